"""dhsa_window_prefill against attention in plain fp64 (paged_plain)."""
import pytest
import torch

import paged_plain
import paper_2510_24606_amd as dhsa

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


def tensors(L, H_q, H_kv, D, dtype, layout, seed=0):
    g = torch.Generator().manual_seed(seed)
    out = []
    for h in (H_q, H_kv, H_kv):
        x = torch.randn((h, L, D), generator=g).to(dtype)
        out.append(x.cuda() if layout == "hld" else x.permute(1, 0, 2).contiguous().cuda().permute(1, 0, 2))
    return out


def check(L, H_q, H_kv, D, dtype, window, sinks, layout="hld", scale=0.0, rows=None):
    print(f"\n[L={L} {H_q}/{H_kv} D={D} {dtype} window={window} sinks={sinks} {layout}]", flush=True)
    Q, K, V = tensors(L, H_q, H_kv, D, dtype, layout)
    O = torch.full_like(Q, float("nan"))
    p = dhsa.problem(Q, K, [0, L], L, scale=scale, V=V)
    dhsa.dhsa_window_prefill(p, Q, K, V, O, window, sinks)
    torch.cuda.synchronize()
    G = H_q // H_kv
    rows = torch.arange(L) if rows is None else rows
    for g in range(H_kv):
        o, _, _, tol, _, _ = paged_plain.attend(Q[g * G:(g + 1) * G, rows.cuda()].cpu(), K[g].cpu(), V[g].cpu(), rows, window, sinks, scale)
        paged_plain.close(O[g * G:(g + 1) * G, rows.cuda()], o, tol, f"kv-head {g}")
    return O


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("L", [1, 2, 15, 16, 17, 31, 33, 63, 64, 65, 127, 129, 300, 1000])
def test_lengths(L, dtype):
    check(L, 4, 2, 64, dtype, max(1, L // 3), 3)
    check(L, 4, 2, 128, dtype, L + 5, 0)


@pytest.mark.parametrize("dtype,D", [(F32, 64), (F32, 128), (BF16, 64), (BF16, 128)])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (2, 700), (5, 3), (31, 0), (32, 1), (33, 64), (64, 4), (100, 65), (128, 129),
                                          (257, 5), (700, 9), (1 << 40, 1 << 40)])
def test_windows_and_sinks(window, sinks, dtype, D):
    check(577, 4, 1, D, dtype, window, sinks, "lhd")


@pytest.mark.parametrize("H_q,H_kv", [(1, 1), (3, 3), (7, 1), (16, 1), (28, 4), (20, 4), (33, 1), (64, 1), (130, 1), (300, 2)])
def test_groups(H_q, H_kv):
    check(131, H_q, H_kv, 64, BF16, 50, 2)
    check(40, H_q, H_kv, 128, F32, 17, 1)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("L,H_q,H_kv,window,sinks", [(5000, 8, 2, 1000, 4), (20000, 4, 1, 3000, 100), (9001, 28, 4, 9001, 0)])
def test_long_prompts(L, H_q, H_kv, window, sinks, dtype):
    """Rows from all over a prompt that fills the chip."""
    rows = torch.unique(torch.cat([torch.arange(40), torch.arange(window - 20, min(window + 20, L)), torch.arange(L - 40, L),
                                   torch.randint(0, L, (150,), generator=torch.Generator().manual_seed(3))]))
    check(L, H_q, H_kv, 128 if dtype == BF16 else 64, dtype, window, sinks, rows=rows)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("L,window,sinks", [(1300, 200, 3), (1700, 1700, 0), (2100, 77, 100), (2400, 500, 1)])
def test_prompts_of_every_tile_height(L, window, sinks, dtype):
    """8 heads of 2 kv-heads: tiles of 16, 32 and 128 rows as the prompt gets longer."""
    rows = torch.unique(torch.cat([torch.arange(20), torch.arange(L - 140, L), torch.randint(0, L, (100,), generator=torch.Generator().manual_seed(L))]))
    for D in (64, 128):
        check(L, 8, 2, D, dtype, window, sinks, "lhd", rows=rows)


def test_scale_and_large_scores():
    check(200, 4, 2, 64, BF16, 90, 2, scale=3.0)        # scores around 200: one key has nearly all of a row
    check(200, 4, 2, 128, F32, 90, 2, scale=0.01)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_scores_that_grow_and_shrink(dtype):
    """The references of the exponentials have to follow scores that climb, and to stay where they fall."""
    L, D = 700, 64
    for order in (1, -1):
        Q, K, V = tensors(L, 2, 1, D, dtype, "hld")
        Q.fill_(1.0)
        K.copy_(((torch.arange(L) if order > 0 else torch.arange(L).flip(0)) * 0.25).to(dtype)[None, :, None].expand(1, L, D))
        O = torch.empty_like(Q)
        dhsa.dhsa_window_prefill(dhsa.problem(Q, K, [0, L], L, scale=0.125), Q, K, V, O, 600, 5)
        torch.cuda.synchronize()
        o, _, _, tol, _, _ = paged_plain.attend(Q.cpu(), K[0].cpu(), V[0].cpu(), torch.arange(L), 600, 5, 0.125)
        paged_plain.close(O, o, tol, f"order {order}")


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_rows_do_not_see_what_is_not_theirs(dtype):
    """Scores of keys behind the row or between the sinks and the window may be anything that is finite."""
    L, D, window, sinks = 400, 64, 33, 2
    Q, K, V = tensors(L, 2, 1, D, dtype, "hld")
    O, O2 = torch.empty_like(Q), torch.empty_like(Q)
    p = dhsa.problem(Q, K, [0, L], L)
    dhsa.dhsa_window_prefill(p, Q, K, V, O, window, sinks)
    row = 200
    K2, V2 = K.clone(), V.clone()
    K2[:, row + 1:] = 1e4
    K2[:, sinks:row - window + 1] = -1e4
    V2[:, row + 1:] = 1e30
    V2[:, sinks:row - window + 1] = -1e30
    dhsa.dhsa_window_prefill(p, Q, K2, V2, O2, window, sinks)
    torch.cuda.synchronize()
    o, _, _, tol, _, _ = paged_plain.attend(Q[:, row:row + 1].cpu(), K[0].cpu(), V[0].cpu(), torch.tensor([row]), window, sinks)
    paged_plain.close(O2[:, row:row + 1], o, tol, "row")
    paged_plain.close(O[:, row:row + 1], o, tol, "row")


def test_equals_the_routed_path_with_everything():
    """Every key in sight: the rows of dhsa_prefill with a budget of all keys (both round probabilities to bf16)."""
    L = 700
    Q, K, V = tensors(L, 8, 2, 128, BF16, "hld")
    O, O2 = torch.empty_like(Q), torch.empty_like(Q)
    B = [0, 100, 250, 400, 700]
    p = dhsa.problem(Q, K, B, L)
    plan, ws = dhsa.alloc(p, B)
    dhsa.dhsa_prefill(p, Q, K, V, B, O2, plan, ws)
    dhsa.dhsa_window_prefill(p, Q, K, V, O, L, 0)
    torch.cuda.synchronize()
    for g in range(2):
        o, _, _, tol, _, _ = paged_plain.attend(Q[4 * g:4 * g + 4].cpu(), K[g].cpu(), V[g].cpu(), torch.arange(L), 0, 0)
        paged_plain.close(O[4 * g:4 * g + 4], o, tol, "window")
        paged_plain.close(O2[4 * g:4 * g + 4], o, tol, "routed")


def test_streams_and_strides():
    """On another stream than the default; rows inside a wider buffer, what lies between them left alone."""
    L, H_q, H_kv, D = 150, 4, 2, 64
    wide = torch.full((L, H_q + 2 * H_kv, D + 64), 7.0, dtype=BF16, device="cuda")
    wide[:, :, :D] = torch.randn((L, H_q + 2 * H_kv, D), generator=torch.Generator().manual_seed(5)).to(BF16).cuda()
    Q, K, V = (wide[:, a:b, :D].permute(1, 0, 2) for a, b in ((0, H_q), (H_q, H_q + H_kv), (H_q + H_kv, H_q + 2 * H_kv)))
    out = torch.full((L, H_q, D + 8), 7.0, dtype=BF16, device="cuda")
    O = out[:, :, :D].permute(1, 0, 2)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        dhsa.dhsa_window_prefill(dhsa.problem(Q, K, [0, L], L, V=V), Q, K, V, O, 40, 3)
    side.synchronize()
    for g in range(H_kv):
        o, _, _, tol, _, _ = paged_plain.attend(Q[2 * g:2 * g + 2].cpu(), K[g].cpu(), V[g].cpu(), torch.arange(L), 40, 3)
        paged_plain.close(O[2 * g:2 * g + 2], o, tol, "O")
    assert (out[:, :, D:] == 7.0).all()


def test_refusals_on_the_device():
    Q, K, V = tensors(20, 4, 2, 64, BF16, "hld")
    O = torch.empty_like(Q)
    p = dhsa.problem(Q, K, [0, 20], 20)
    for bad in (dict(Q=Q[:, :19]), dict(K=K.float()), dict(V=V[:1]), dict(O=O.float()), dict(K=K[:1].expand(2, 20, 64)),
                dict(O=torch.empty((4, 64, 20), dtype=BF16, device="cuda").transpose(1, 2))):
        t = dict(Q=Q, K=K, V=V, O=O)
        t.update(bad)
        with pytest.raises(ValueError):
            dhsa.dhsa_window_prefill(p, t["Q"], t["K"], t["V"], t["O"], 5, 0)
    with pytest.raises(dhsa.DhsaError):
        dhsa.dhsa_window_prefill(p, Q, K, V, O, 0, 0)
