"""The paged cache at what its callers may hand over by mistake or in passing."""
import pytest
import torch

import paged_plain
import paper_2510_24606_amd as dhsa
from test_gpu_paged import Batch

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


@pytest.mark.parametrize("dtype,D", [(F32, 64), (F32, 128), (BF16, 64), (BF16, 128)])
@pytest.mark.parametrize("lens,row", [([(1, 40), (1, 30)], 0), ([(1, 9000), (1, 20)], 0), ([(1, 20), (3, 9000)], 2),
                                      ([(70, 90), (3, 40)], 33), ([(60, 9000), (2, 50)], 7), ([(200, 300)], 199)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (50, 3)])
def test_a_row_that_is_not_a_number(lens, row, window, sinks, dtype, D):
    """It says so in O, in lse and in the weights of the keys that it sees, however long the cache is; nothing else does."""
    b = Batch(lens, 4, 2, D, dtype, 16, window=window, sinks=sinks)
    W, W2 = b.new_weights(), b.new_weights()
    before = W.clone()
    O, lse = b.attend(W, 0.0)
    Q = b.Q.clone()
    b.Q[1, row, D // 2] = float("nan")                  # one head of the first kv-head
    O2, lse2 = b.attend(W2, 0.0)
    assert torch.isnan(O2[1, row]).all() and torch.isnan(lse2[1, row])
    for s, (n, kv) in enumerate(lens):
        page, slot = (x.cuda() for x in b.slots(s))
        sees = torch.zeros(kv, dtype=torch.bool)
        if b.starts[s] <= row < b.starts[s + 1]:
            sees = paged_plain.sees(torch.tensor([kv - n + row - b.starts[s]]), kv, window, sinks)[0]
        got = W2[page, :, slot]
        assert torch.equal(torch.isnan(got[:, 0]).cpu(), sees) and not torch.isnan(got[:, 1]).any()
        W[page, :, slot] = torch.where(torch.isnan(got), W[page, :, slot], got)
    b.Q, O2[1, row], lse2[1, row] = Q, O[1, row], lse[1, row]
    b.check(O2, lse2, before, W, 0.0)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("L", [50, 700, 5000])
def test_a_row_of_a_prompt_that_is_not_a_number(L, dtype):
    g = torch.Generator().manual_seed(L)
    Q, K, V = (torch.randn((h, L, 64), generator=g).to(dtype).cuda() for h in (8, 2, 2))
    O, O2 = torch.empty_like(Q), torch.empty_like(Q)
    p = dhsa.problem(Q, K, [0, L], L)
    dhsa.dhsa_window_prefill(p, Q, K, V, O, 100, 2)
    Q[3, L // 2, 5] = float("nan")
    dhsa.dhsa_window_prefill(p, Q, K, V, O2, 100, 2)
    torch.cuda.synchronize()
    assert torch.isnan(O2[3, L // 2]).all()
    O2[3, L // 2] = O[3, L // 2]
    rows = torch.unique(torch.cat([torch.arange(max(0, L // 2 - 140), min(L, L // 2 + 140)), torch.arange(20)]))
    for h in range(2):
        q = Q[4 * h:4 * h + 4, rows.cuda()].nan_to_num(0.0).cpu()
        o, _, _, tol, _, _ = paged_plain.attend(q, K[h].cpu(), V[h].cpu(), rows, 100, 2)
        got = O2[4 * h:4 * h + 4, rows.cuda()].cpu()
        if h == 0:
            at = int((rows == L // 2).nonzero())
            got[3, at] = o[3, at].to(dtype)
        paged_plain.close(got, o, tol, f"kv-head {h}")


@pytest.mark.parametrize("dtype,D", [(F32, 64), (BF16, 128)])
def test_tokens_behind_the_table_are_left_out(dtype, D):
    """A sequence that is said to be longer than its table: the tokens that fit go where they belong, the slots before them and the
    weights there stay, the other tokens go nowhere."""
    for n, kv, cap in ((10, 69, 64), (10, 64, 64), (3, 80, 64), (64, 70, 64), (100, 90, 64), (1, 65, 64), (5, (1 << 31) - 1, 64)):
        b = Batch([(2, 20), (n, cap), (1, 7)], 4, 2, D, dtype, 16)
        assert b.table.shape[1] * 16 == cap
        b.K.nan_to_num_(3.0); b.V.nan_to_num_(3.0)
        b.kv_len[1] = kv
        Kn, Vn = (torch.randn((2, b.T, D), generator=b.g).to(dtype).cuda() for _ in range(2))
        W = b.new_weights()
        K, V, W2 = b.K.clone(), b.V.clone(), W.clone()
        dhsa.dhsa_paged_append(b.prob, Kn, Vn, b.K, b.V, b.table, b.q_start, b.kv_len, W)
        torch.cuda.synchronize()
        table = b.table.cpu()
        for s, (rows, end) in enumerate(((2, 20), (n, kv), (1, 7))):
            for i in range(rows):
                slot = end - rows + i
                if 0 <= slot < cap:
                    page, at = int(table[s, slot // 16]), slot % 16
                    K[page, :, at], V[page, :, at] = Kn[:, b.starts[s] + i], Vn[:, b.starts[s] + i]
                    W2[page, :, at] = 0.0
        assert torch.equal(b.K, K) and torch.equal(b.V, V) and torch.equal(W, W2), (n, kv)


@pytest.mark.parametrize("dtype,D", [(F32, 64), (BF16, 128)])
@pytest.mark.parametrize("n,over", [(3, 2), (10, 3), (40, 25), (150, 60), (30, 40), (6, (1 << 31) - 65)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (20, 3)])
def test_rows_behind_the_table_keep_their_places(n, over, window, sinks, dtype, D):
    """Rows of such tokens attend to the slots that there are, from where they are; so do rows that are said to end behind T."""
    cap = 64
    b = Batch([(2, 20), (n, cap)], 4, 2, D, dtype, 16, window=window, sinks=sinks)
    b.kv_len[1] = cap + over
    pos = cap + over - n + torch.arange(n, dtype=torch.int64)
    for far in (0, 9):
        if far:
            if over > 1000:
                continue
            b.q_start[2] += far                        # nine more rows than there are, and as many more tokens
            b.kv_len[1] += far
        W = b.new_weights()
        O, lse = b.attend(W, 0.0)
        for g in range(2):
            rows = slice(2, 2 + n)
            o, z, got, t_o, t_z, t_w = paged_plain.attend(b.Q[2 * g:2 * g + 2, rows].cpu(), b.kc[1][g], b.vc[1][g], pos, window, sinks)
            paged_plain.close(O[2 * g:2 * g + 2, rows], o, t_o, "O")
            paged_plain.close(lse[2 * g:2 * g + 2, rows], z, t_z, "lse")
            page, slot = b.slots(1)
            paged_plain.close(W[page, g, slot], got, t_w, "weights")


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_weights_in_a_workspace_of_more_tokens(dtype):
    """Its room for scores is too small for those of all sequences; nothing behind it is written."""
    b = Batch([(1, 16000)] * 20, 32, 2, 64, dtype, 16, window=9000, sinks=5)
    more = dhsa.dhsa_paged.from_buffer_copy(b.prob)
    more.T = 22 if dtype == BF16 else 41                # 17 (33) rows a kv-head and sequence in the mean
    full, size = dhsa.dhsa_paged_workspace_bytes(b.prob), dhsa.dhsa_paged_workspace_bytes(more)
    if dtype == F32:
        size = min(size, dhsa.dhsa_paged_workspace_bytes(more, False) + 8 * 32 * more.T + 256)
    assert size < full
    whole = torch.full((size + 4096,), 77, dtype=torch.uint8, device="cuda")
    W = b.new_weights()
    before = W.clone()
    b.check(*b.attend(W, 0.5, ws=whole[:size]), before, W, 0.5)
    assert (whole[size:] == 77).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_strides_of_a_single_one(dtype):
    """One sequence, token, head and page: their strides may say anything."""
    from test_paged_edges_host import odd
    b = Batch([(1, 37)], 1, 1, 64, dtype, 48, spare=0)
    Kn, Vn = (odd(torch.randn((1, 1, 64), generator=b.g).to(dtype).cuda()) for _ in range(2))
    b.K, b.V, b.Q, b.table = odd(b.K), odd(b.V), odd(b.Q), odd(b.table)
    b.prob = dhsa.paged_problem(b.K, b.V, b.table, 1, 1)
    W = odd(b.new_weights())
    dhsa.dhsa_paged_append(b.prob, Kn, Vn, b.K, b.V, b.table, b.q_start, b.kv_len, W)
    b.kc[0][:, 36], b.vc[0][:, 36] = Kn[:, 0].cpu(), Vn[:, 0].cpu()
    before = W.clone()
    assert (W[0, 0, 36] == 0).all()
    b.check(*b.attend(W, 1.0), before, W, 1.0)
