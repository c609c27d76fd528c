"""The paged cache (append, attend with and without weights, evict) against plain fp64 on the CPU (paged_plain)."""
import pytest
import torch

import paged_plain
import paper_2510_24606_amd as dhsa

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


class Batch:
    """Sequences of (new tokens, tokens) in pages in any order, the rest of the pool NaN."""

    def __init__(self, lens, H_q, H_kv, D, dtype, page, layout="hld", seed=0, window=0, sinks=0, spare=2, max_pages=None, pool="phsd",
                 extra_rows=0, scale=0.0):
        self.g = torch.Generator().manual_seed(seed)
        self.lens, self.H_q, self.H_kv, self.D, self.dtype, self.page = lens, H_q, H_kv, D, dtype, page
        self.window, self.sinks, self.layout, self.scale = window, sinks, layout, scale
        need = [-(-kv // page) for _, kv in lens]
        n = sum(need) + spare
        order = torch.randperm(n, generator=self.g).to(torch.int32)
        width = max(need + [1]) if max_pages is None else max_pages
        self.table = torch.full((len(lens), width), -7, dtype=torch.int32)
        at = 0
        for s, c in enumerate(need):
            self.table[s, :c] = order[at:at + c]
            at += c
        starts = [0]
        for q, _ in lens:
            starts.append(starts[-1] + q)
        self.starts, self.T = starts, starts[-1] + extra_rows
        self.kc = [torch.randn((H_kv, kv, D), generator=self.g).to(dtype) for _, kv in lens]
        self.vc = [torch.randn((H_kv, kv, D), generator=self.g).to(dtype) for _, kv in lens]
        K, V = (torch.full((n, H_kv, page, D), float("nan"), dtype=dtype) for _ in range(2))
        for s, (_, kv) in enumerate(lens):
            for i in range(need[s]):
                m = min(page, kv - i * page)
                K[self.table[s, i], :, :m] = self.kc[s][:, i * page:i * page + m]
                V[self.table[s, i], :, :m] = self.vc[s][:, i * page:i * page + m]
        if pool == "pshd":
            self.K, self.V = (x.permute(0, 2, 1, 3).contiguous().cuda().permute(0, 2, 1, 3) for x in (K, V))
        else:
            self.K, self.V = K.cuda(), V.cuda()
        Q = torch.randn((H_q, self.T, D), generator=self.g).to(dtype)
        self.Q = Q.cuda() if layout == "hld" else Q.permute(1, 0, 2).contiguous().cuda().permute(1, 0, 2)
        self.table = self.table.cuda()
        self.q_start = torch.tensor(starts, dtype=torch.int32).cuda()
        self.kv_len = torch.tensor([kv for _, kv in lens], dtype=torch.int32).cuda()
        self.prob = dhsa.paged_problem(self.K, self.V, self.table, H_q, self.T, window=window, sinks=sinks, scale=scale)

    def new_weights(self):
        return torch.rand((self.K.shape[0], self.H_kv, self.page), generator=self.g).cuda()

    def attend(self, weights=None, decay=1.0, ws=None):
        O = torch.full_like(self.Q, 7.0)
        lse = torch.full((self.H_q, self.T), 7.0, dtype=F32, device="cuda")
        ws = dhsa.alloc_paged(self.prob) if ws is None else ws
        ws.fill_(255)                                           # nothing in it has to be set
        dhsa.dhsa_paged_attend(self.prob, self.Q, self.K, self.V, self.table, self.q_start, self.kv_len, O, ws, lse=lse, weights=weights,
                               decay=decay)
        torch.cuda.synchronize()
        return O, lse

    def slots(self, s):
        """(page, slot) of the tokens of sequence s, on the CPU; page -1 where the table has none"""
        j = torch.arange(self.lens[s][1])
        return self.table[s].cpu().long()[j // self.page], j % self.page

    def check(self, O, lse, before=None, weights=None, decay=1.0, bad=()):
        """bad: (sequence, page index) pairs that the table has no page for"""
        G, n_s = self.H_q // self.H_kv, len(self.lens)
        after = None if weights is None else weights.cpu()
        expect = None if weights is None else before.cpu().double()
        tol_w = None if weights is None else torch.zeros_like(expect)
        for s, (n, kv) in enumerate(self.lens):
            rows = slice(self.starts[s], self.starts[s + 1])
            valid = torch.ones(kv, dtype=torch.bool)
            for bs, bp in bad:
                if bs == s:
                    valid[bp * self.page:(bp + 1) * self.page] = False
            page, slot = self.slots(s)
            for g in range(self.H_kv):
                q = self.Q[g * G:(g + 1) * G, rows].cpu()
                if n:
                    o, z, got, t_o, t_z, t_w = paged_plain.attend(q, self.kc[s][g], self.vc[s][g], torch.arange(kv - n, kv), self.window, self.sinks,
                                                                  self.scale, valid)
                    paged_plain.close(O[g * G:(g + 1) * G, rows], o, t_o, f"O of sequence {s}, kv-head {g}")
                    paged_plain.close(lse[g * G:(g + 1) * G, rows], z, t_z, f"lse of sequence {s}, kv-head {g}")
                else:
                    got, t_w = torch.zeros(kv, dtype=torch.float64), torch.zeros(kv, dtype=torch.float64)
                if weights is not None:
                    p, j = page[valid], slot[valid]
                    old = expect[p, g, j]
                    expect[p, g, j] = decay * old + got[valid]
                    tol_w[p, g, j] = t_w[valid] + 2.0 ** -23 * (decay * old + got[valid])
        if weights is not None:
            paged_plain.close(after, expect, tol_w, "weights")
        assert (O[:, self.starts[-1]:] == 7.0).all() and (lse[:, self.starts[-1]:] == 7.0).all()


def run(lens, H_q=4, H_kv=2, D=64, dtype=BF16, page=16, weights=False, decay=1.0, **kw):
    print(f"\n[{lens if len(lens) < 9 else len(lens)} {H_q}/{H_kv} D={D} {dtype} page={page} {kw}]", flush=True)
    b = Batch(lens, H_q, H_kv, D, dtype, page, **kw)
    W = b.new_weights() if weights else None
    before = W.clone() if weights else None
    O, lse = b.attend(W, decay)
    b.check(O, lse, before, W, decay)
    return b, O, lse


RAGGED = [(1, 100), (0, 50), (3, 3), (17, 40), (1, 1), (0, 0), (64, 64), (5, 129)]


@pytest.mark.parametrize("dtype,D", [(F32, 64), (F32, 128), (BF16, 64), (BF16, 128)])
@pytest.mark.parametrize("page", [1, 3, 16, 17, 64, 1000])
def test_pages(page, dtype, D):
    run(RAGGED, D=D, dtype=dtype, page=page, weights=True)
    run(RAGGED, D=D, dtype=dtype, page=page, weights=True, window=20, sinks=2, pool="pshd", layout="lhd", extra_rows=3)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("kv", [1, 2, 15, 16, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 257, 1000, 5000])
def test_single_tokens(kv, dtype):
    run([(1, kv)], 8, 2, 128, dtype, 16, weights=True)
    run([(1, kv), (1, 1), (1, (kv + 1) // 2)], 8, 1, 64, dtype, 64, weights=True, window=max(1, kv // 3), sinks=1)


@pytest.mark.parametrize("lens", [[(8, 300)], [(16, 16)], [(33, 2000)], [(200, 200)], [(300, 1111)], [(1, 3000), (250, 700)], [(129, 130), (2, 5000)]])
@pytest.mark.parametrize("G", [1, 4, 7])
def test_chunks(lens, G):
    run(lens, 2 * G, 2, 128, BF16, 16, weights=True)
    run(lens, G, 1, 64, F32, 24, weights=True, window=100, sinks=5)


@pytest.mark.parametrize("H_q,H_kv", [(1, 1), (3, 3), (16, 1), (17, 1), (40, 1), (130, 2), (36, 12)])
def test_groups(H_q, H_kv):
    run([(1, 200), (3, 90)], H_q, H_kv, 64, BF16, 16, weights=True)
    run([(1, 200), (3, 90)], H_q, H_kv, 128, F32, 16, weights=True, window=33, sinks=1)


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (7, 200), (32, 3), (64, 0), (100, 33), (1 << 40, 5)])
def test_windows(window, sinks):
    run([(1, 700), (40, 300), (9, 9), (70, 71)], window=window, sinks=sinks, weights=True, decay=0.5)


@pytest.mark.parametrize("n_seq", [63, 64, 65, 130, 300])
def test_many_sequences(n_seq):
    """More sequences than a wave looks at at once, some of them empty, one much longer than the others."""
    g = torch.Generator().manual_seed(n_seq)
    lens = []
    for s in range(n_seq):
        kv = int(torch.randint(0, 60, (1,), generator=g))
        lens.append((min(kv, int(torch.randint(0, 3, (1,), generator=g))), kv))
    lens[n_seq // 2] = (2, 4000)
    lens[-1] = (1, 77)
    run(lens, 4, 2, 64, BF16, 16, weights=True)


@pytest.mark.parametrize("dtype,D", [(F32, 64), (F32, 128), (BF16, 64), (BF16, 128)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (60, 3)])
def test_few_rows_in_the_mean(window, sinks, dtype, D):
    """Small tiles, several of them a sequence: scores of 24 rows are kept, those of 80 are made again for the weights."""
    run([(1, 50)] * 9 + [(6, 500)] + [(1, 33)] * 3, 8, 2, D, dtype, 16, weights=True, window=window, sinks=sinks)
    run([(1, 40)] * 30 + [(20, 300), (2, 31)], 8, 2, D, dtype, 24, weights=True, decay=0.5, window=window, sinks=sinks)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_scores_that_do_not_fit(dtype):
    """The workspace keeps scores for as many rows as a sequence has in the mean: of one with eight times as many, and of those
    behind it, they are made again."""
    run([(1, 16)] * 5 + [(8, 2000)] + [(1, 16)] * 25, 8, 2, 64, dtype, 16, weights=True)
    run([(8, 2000)] + [(1, 16)] * 30, 4, 1, 128, dtype, 64, weights=True, window=300, sinks=70)


def test_long_and_short_together():
    """One conversation is cut into many pieces beside short ones; sums over 40000 keys."""
    run([(1, 9), (1, 40000), (2, 70), (0, 10), (1, 1000)], 4, 1, 128, BF16, 64, weights=True)
    run([(1, 9), (1, 20000), (2, 70)], 4, 2, 64, F32, 48, weights=True)


def test_rows_without_keys():
    """More new tokens than the sequence is said to have: the first of them see nothing."""
    b = Batch([(6, 20), (3, 3)], 4, 2, 64, BF16, 16)
    b.kv_len = torch.tensor([2, 3], dtype=torch.int32).cuda()
    W = b.new_weights()
    before = W.clone()
    O, lse = b.attend(W, 0.0)
    assert (O[:, :4] == 0).all() and torch.isinf(lse[:, :4]).all() and (lse[:, :4] < 0).all()
    for g in range(2):
        o, z, got, t_o, t_z, t_w = paged_plain.attend(b.Q[2 * g:2 * g + 2, 4:6].cpu(), b.kc[0][g, :2], b.vc[0][g, :2], torch.arange(2), 0, 0)
        paged_plain.close(O[2 * g:2 * g + 2, 4:6], o, t_o, "O")
        paged_plain.close(lse[2 * g:2 * g + 2, 4:6], z, t_z, "lse")
        paged_plain.close(W[b.table[0, 0], g, :2], got, t_w, "weights")
    assert torch.equal(W[b.table[0, 0].long(), :, 2:], before[b.table[0, 0].long(), :, 2:])     # slots behind the tokens


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("value", [-1, 1 << 30, -(1 << 31)])
def test_pages_that_are_none(value, dtype):
    """A page outside the pool is left out, in the middle, at the end and as the only one."""
    b = Batch([(3, 100), (1, 30), (40, 90)], 4, 2, 64, dtype, 16)
    bad = [(0, 2), (0, 6), (1, 0), (1, 1), (2, 0)]
    for s, i in bad:
        b.table[s, i] = value
    W = b.new_weights()
    before = W.clone()
    O, lse = b.attend(W, 0.25)
    b.check(O, lse, before, W, 0.25, bad)
    assert (O[:, 3] == 0).all()                                                # the only pages of sequence 1
    Kn = torch.randn((2, b.T, 64), device="cuda").to(dtype)
    K0, V0 = b.K.clone(), b.V.clone()
    dhsa.dhsa_paged_append(b.prob, Kn, Kn, b.K, b.V, b.table, b.q_start, b.kv_len, W)
    torch.cuda.synchronize()
    for x, y in ((b.K, K0), (b.V, V0)):
        changed = (x.view(torch.uint8) != y.view(torch.uint8)).flatten(1).any(1).nonzero().flatten().tolist()
        ok = set(int(b.table[0, i]) for i in range(7)) | set(int(b.table[2, i]) for i in range(6))
        assert changed and set(changed) <= ok - {value}


def test_lengths_that_do_not_fit():
    """Starts and lengths out of range are clamped: nothing outside the arrays is touched."""
    b = Batch([(2, 30), (2, 30)], 4, 2, 64, BF16, 16, extra_rows=4)
    b.q_start = torch.tensor([-5, 2, 1 << 30], dtype=torch.int32).cuda()
    b.kv_len = torch.tensor([-4, 1 << 30], dtype=torch.int32).cuda()
    b.K.nan_to_num_(0.0); b.V.nan_to_num_(0.0)
    O, lse = b.attend()
    assert (O[:, :2] == 0).all() and torch.isfinite(O.float()).all()
    b.q_start = torch.tensor([4, 2, 0], dtype=torch.int32).cuda()
    O, lse = b.attend()
    assert (O == 7.0).all()
    Kn = torch.zeros((2, b.T, 64), dtype=BF16, device="cuda")
    b.q_start = torch.tensor([0, 8, 8], dtype=torch.int32).cuda()
    b.kv_len = torch.tensor([3, -1], dtype=torch.int32).cuda()
    dhsa.dhsa_paged_append(b.prob, Kn, Kn, b.K, b.V, b.table, b.q_start, b.kv_len)
    torch.cuda.synchronize()
    page = int(b.table[0, 0])
    assert (b.K[page, :, :3] == 0).all() and not (b.K[page, :, 3:] == 0).all()


def test_rows_that_are_nobodys():
    """Rows before the first sequence and behind the last one stay as they were, also where others are cut into pieces and the
    workspace holds what an earlier call left."""
    b = Batch([(2, 3000), (1, 40)], 4, 2, 64, BF16, 16, extra_rows=2)
    ws = dhsa.alloc_paged(b.prob)
    O, lse = b.attend(ws=ws)
    b.check(O, lse)
    dhsa.dhsa_paged_attend(b.prob, b.Q, b.K, b.V, b.table, b.q_start, b.kv_len, O, ws, lse=lse)      # leaves its states in ws
    b.q_start = torch.tensor([1, 2, 3], dtype=torch.int32).cuda()
    O2, lse2 = torch.full_like(b.Q, 7.0), torch.full((4, b.T), 7.0, device="cuda")
    dhsa.dhsa_paged_attend(b.prob, b.Q, b.K, b.V, b.table, b.q_start, b.kv_len, O2, ws, lse=lse2)
    torch.cuda.synchronize()
    for x in (O2, lse2):
        assert (x[:, :1] == 7.0).all() and (x[:, 3:] == 7.0).all() and not (x[:, 1:3] == 7.0).all()
    for g in range(2):
        o, z, _, t_o, t_z, _ = paged_plain.attend(b.Q[2 * g:2 * g + 2, 1:2].cpu(), b.kc[0][g], b.vc[0][g], torch.tensor([2999]), 0, 0)
        paged_plain.close(O2[2 * g:2 * g + 2, 1:2], o, t_o, "O")
        paged_plain.close(lse2[2 * g:2 * g + 2, 1:2], z, t_z, "lse")


def test_a_pool_beyond_32_bits():
    """Pages whose offsets pass 2^32 bytes and 2^31 elements."""
    page, H_kv, D = 64, 2, 128
    per = page * H_kv * D * 2
    n = ((1 << 32) + (64 << 20)) // per + 8
    K = torch.zeros((n, H_kv, page, D), dtype=BF16, device="cuda")
    V = torch.zeros((n, H_kv, page, D), dtype=BF16, device="cuda")
    b = Batch([(5, 200), (1, 100)], 4, 2, D, BF16, page)
    place = torch.tensor([n - 1, n - 5, 3, n - 2, n // 2 + 1, n - 9], dtype=torch.int32)
    table = b.table.clone().fill_(-1)
    at = 0
    for s, (_, kv) in enumerate(b.lens):
        for i in range(-(-kv // page)):
            K[place[at]], V[place[at]] = b.K[b.table[s, i]], b.V[b.table[s, i]]
            table[s, i] = place[at]
            at += 1
    b.K, b.V, b.table = K, V, table
    b.prob = dhsa.paged_problem(K, V, table, 4, b.T)
    W = torch.zeros((n, H_kv, page), device="cuda")
    O, lse = b.attend(W, 0.0)
    b.check(O, lse, torch.zeros_like(W), W, 0.0)
    Kn = torch.randn((2, b.T, D), device="cuda").to(BF16)
    dhsa.dhsa_paged_append(b.prob, Kn, Kn, b.K, b.V, b.table, b.q_start, b.kv_len, W)
    torch.cuda.synchronize()
    assert torch.equal(K[n - 2, :, 195 % 64:200 % 64], Kn[:, :5]) and torch.equal(V[n - 9, :, 99 % 64], Kn[:, 5])
    assert (W[n - 2, :, 3:8] == 0).all() and (W[n - 2, :, :3] > 0).all()


def test_a_contiguous_cache_is_one_page():
    """dhsa_decode_step with a budget of everything, over the same cache: the same row."""
    L, H_q, H_kv, D = 900, 8, 2, 128
    g = torch.Generator().manual_seed(4)
    Q, K, V = (torch.randn((h, L, D), generator=g).to(BF16).cuda() for h in (H_q, H_kv, H_kv))
    B = [0, 300, 900]
    p = dhsa.problem(Q, K, B, L)
    row = dhsa.dhsa_decode_step(p, Q, K, V, B, dhsa.alloc_decode(p, 2, L), 2, L)
    table = torch.zeros((1, 1), dtype=torch.int32, device="cuda")
    pp = dhsa.paged_problem(K[None], V[None], table, H_q, 1)
    O = torch.empty((H_q, 1, D), dtype=BF16, device="cuda")
    dhsa.dhsa_paged_attend(pp, Q[:, -1:], K[None], V[None], table, torch.tensor([0, 1], dtype=torch.int32, device="cuda"),
                           torch.tensor([L], dtype=torch.int32, device="cuda"), O, dhsa.alloc_paged(pp))
    torch.cuda.synchronize()
    for h in range(H_kv):
        o, _, _, tol, _, _ = paged_plain.attend(Q[4 * h:4 * h + 4, -1:].cpu(), K[h].cpu(), V[h].cpu(), torch.tensor([L - 1]), 0, 0)
        paged_plain.close(O[4 * h:4 * h + 4], o, tol, "paged")
        paged_plain.close(row[4 * h:4 * h + 4, None], o, tol, "decode_step")


def test_shared_pages():
    """Two sequences that begin with the same pages (read only)."""
    b = Batch([(2, 100), (3, 100)], 4, 2, 64, BF16, 16)
    b.table[1, :5] = b.table[0, :5]
    for x in (b.kc, b.vc):
        x[1][:, :80] = x[0][:, :80]
    O, lse = b.attend()
    b.check(O, lse)


def test_two_calls_share_a_workspace_and_streams():
    """Calls on one stream one after another through one workspace; another stream."""
    side = torch.cuda.Stream()
    a, b = Batch([(1, 3000), (1, 50)], 4, 2, 64, BF16, 16, seed=1), Batch([(1, 20), (1, 4000)], 4, 2, 64, BF16, 16, seed=2)
    ws = dhsa.alloc_paged(a.prob)
    outs = []
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for x in (a, b, a):
            O, lse = torch.full_like(x.Q, 7.0), torch.full((4, x.T), 7.0, device="cuda")
            dhsa.dhsa_paged_attend(x.prob, x.Q, x.K, x.V, x.table, x.q_start, x.kv_len, O, ws, lse=lse)
            outs.append((x, O, lse))
    side.synchronize()
    for x, O, lse in outs:
        x.check(O, lse)
    assert torch.equal(outs[0][1], outs[2][1])


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_results_do_not_change(dtype):
    """The same bits call after call: no order of anything hangs on timing."""
    b = Batch([(1, 3000), (70, 500), (1, 50)], 8, 2, 64, dtype, 16)
    first = None
    for _ in range(4):
        W = torch.ones((b.K.shape[0], 2, 16), device="cuda")
        O, lse = b.attend(W, 0.5)
        got = (O.clone(), lse.clone(), W)
        if first is not None:
            assert all(torch.equal(x, y) for x, y in zip(first, got))
        first = got


# ---- append ----

@pytest.mark.parametrize("dtype,D", [(F32, 64), (F32, 128), (BF16, 64), (BF16, 128)])
@pytest.mark.parametrize("page", [1, 5, 16, 64])
@pytest.mark.parametrize("layout", ["hld", "lhd"])
def test_append(page, layout, dtype, D):
    b = Batch(RAGGED, 4, 2, D, dtype, page, pool="pshd" if layout == "lhd" else "phsd", extra_rows=2)
    W = b.new_weights()
    Kn, Vn = (torch.randn((2, b.T, D) if layout == "hld" else (b.T, 2, D), generator=b.g).to(dtype).cuda() for _ in range(2))
    if layout == "lhd":
        Kn, Vn = Kn.permute(1, 0, 2), Vn.permute(1, 0, 2)
    K, V, W1 = b.K.clone(), b.V.clone(), W.clone()
    for s, (n, kv) in enumerate(b.lens):
        p, j = (x[kv - n:].cuda() for x in b.slots(s))
        rows = slice(b.starts[s], b.starts[s + 1])
        K[p, :, j], V[p, :, j] = Kn[:, rows].transpose(0, 1), Vn[:, rows].transpose(0, 1)
        W1[p, :, j] = 0
    dhsa.dhsa_paged_append(b.prob, Kn, Vn, b.K, b.V, b.table, b.q_start, b.kv_len, W)
    torch.cuda.synchronize()
    bits = torch.int32 if dtype == F32 else torch.int16
    assert torch.equal(b.K.view(bits), K.view(bits)) and torch.equal(b.V.view(bits), V.view(bits)) and torch.equal(W, W1)


def test_append_many():
    lens = [(3, 10 + i % 40) for i in range(200)]
    b = Batch(lens, 4, 2, 64, BF16, 16)
    Kn = torch.randn((2, b.T, 64), generator=b.g).to(BF16).cuda()
    dhsa.dhsa_paged_append(b.prob, Kn, Kn, b.K, b.V, b.table, b.q_start, b.kv_len)
    torch.cuda.synchronize()
    for s, (n, kv) in enumerate(lens):
        p, j = (x[kv - n:].cuda() for x in b.slots(s))
        assert torch.equal(b.K[p, :, j].transpose(0, 1), Kn[:, b.starts[s]:b.starts[s + 1]]), s


# ---- evict ----

def evict_plain(w, kv, keep, first, recent):
    """Slots that stay of one head: w fp32 [kv]"""
    if kv <= keep:
        return torch.arange(kv)
    middle = w[first:kv - recent].clone().double()
    middle = torch.where(torch.isnan(middle), torch.tensor(float("-inf"), dtype=torch.float64), middle)
    nan = torch.isnan(w[first:kv - recent])
    order = sorted(range(len(middle)), key=lambda i: (bool(nan[i]), -float(middle[i]), i))
    best = torch.tensor(order[:keep - first - recent], dtype=torch.long) + first
    return torch.sort(torch.cat([torch.arange(first), best, torch.arange(kv - recent, kv)]))[0]


def evict_check(b, W, keep, first, recent, in_place):
    n_s, page = len(b.lens), b.page
    K0, V0, W0, old = b.K.clone(), b.V.clone(), W.clone(), b.table.clone()
    out, kv_out = None, torch.full_like(b.kv_len, -5)
    if not in_place:
        used = set(int(x) for x in old.flatten())
        free = [i for i in range(b.K.shape[0]) if i not in used]
        out = torch.full_like(old, -9)
        for s, (_, kv) in enumerate(b.lens):
            for i in range(-(-min(kv, keep) // page)):
                out[s, i] = free.pop()
    idx = torch.full((n_s, b.H_kv, keep), -8, dtype=torch.int32, device="cuda")
    ws = dhsa.alloc_evict(b.prob, keep)
    ws.fill_(255)
    kv_arg = b.kv_len if in_place else kv_out                  # in place: the lengths too
    lens = b.kv_len.clone()
    dhsa.dhsa_paged_evict(b.prob, b.K, b.V, W, b.table, b.kv_len, keep, first, recent, ws, kv_arg, table_out=out, idx=idx)
    torch.cuda.synchronize()
    assert torch.equal(kv_arg, torch.clamp(lens, max=keep))
    to_table = (old if in_place else out).cpu().long()
    K1, V1, W1 = K0.clone(), V0.clone(), W0.clone()
    for s, (_, kv) in enumerate(b.lens):
        p, j = b.slots(s)
        for g in range(b.H_kv):
            kept = evict_plain(W0[p, g, j].cpu(), kv, keep, first, recent)
            m = len(kept)
            assert torch.equal(idx[s, g, :m].cpu().long(), kept), (s, g)
            assert (idx[s, g, m:] == -1).all()
            t = torch.arange(m)
            tp, tj = to_table[s][t // page].cuda(), (t % page).cuda()
            for x, y in ((K1, K0), (V1, V0), (W1, W0)):
                x[tp, g, tj] = y[p[kept].cuda(), g, j[kept].cuda()]
    bits = torch.int32 if b.dtype == F32 else torch.int16
    assert torch.equal(b.K.view(bits), K1.view(bits)) and torch.equal(b.V.view(bits), V1.view(bits))
    assert torch.equal(W.view(torch.int32), W1.view(torch.int32))


EVICT_LENS = [(0, 500), (0, 30), (0, 0), (0, 41), (0, 40), (0, 1300)]


@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("dtype,D,page", [(F32, 64, 16), (F32, 128, 7), (BF16, 64, 64), (BF16, 128, 1)])
@pytest.mark.parametrize("keep,first,recent", [(40, 4, 10), (40, 0, 0), (40, 40, 0), (40, 0, 40), (40, 10, 30), (1, 0, 0), (1, 1, 0), (1400, 3, 3),
                                               (499, 0, 1)])
def test_evict(keep, first, recent, dtype, D, page, in_place):
    print(f"\n[keep={keep} first={first} recent={recent} {dtype} D={D} page={page}]", flush=True)
    b = Batch(EVICT_LENS, 4, 2, D, dtype, page, spare=2400 // page + 20, pool="pshd" if page == 7 else "phsd")
    W = (torch.randn((b.K.shape[0], 2, page), generator=b.g) * 2).exp().cuda()
    evict_check(b, W, keep, first, recent, in_place)


def test_evict_ties_and_odd_weights():
    """Equal weights (a lower slot stays), zeros of both signs, infinities, negative ones and NaN."""
    for seed in range(3):
        b = Batch([(0, 700), (0, 300)], 4, 2, 64, BF16, 16, seed=seed)
        values = torch.tensor([0.0, -0.0, 1.0, 1.0, float("inf"), float("-inf"), float("nan"), -float("nan"), 1e-45, -1e-45, 3e38, -2.0])
        W = values[torch.randint(0, len(values), (b.K.shape[0], 2, 16), generator=b.g)].cuda()
        evict_check(b, W, 100, 2, 5, True)
        b = Batch([(0, 700)], 4, 2, 64, BF16, 16, seed=seed)
        evict_check(b, torch.full((b.K.shape[0], 2, 16), float("nan") if seed == 0 else 2.5, device="cuda"), 300, 0, 1, True)


@pytest.mark.parametrize("kv,keep", [(40000, 5000), (70000, 69990), (20000, 1)])
def test_evict_long(kv, keep):
    b = Batch([(0, kv)], 2, 1, 64, BF16, 64)
    W = torch.rand((b.K.shape[0], 1, 64), generator=b.g).pow(8).cuda()
    evict_check(b, W, keep, min(4, keep), 0 if keep == 1 else 700, True)


def test_evict_without_a_page():
    """Slots whose page is none go first; nothing is written outside the pool."""
    b = Batch([(0, 200)], 4, 2, 64, BF16, 16)
    b.table[0, 3] = -1
    W = torch.rand((b.K.shape[0], 2, 16), generator=b.g).cuda()
    kv_out, idx = torch.zeros_like(b.kv_len), torch.zeros((1, 2, 100), dtype=torch.int32, device="cuda")
    K0, W0 = b.K.clone(), W.clone()
    dhsa.dhsa_paged_evict(b.prob, b.K, b.V, W, b.table, b.kv_len, 100, 0, 0, dhsa.alloc_evict(b.prob, 100), kv_out, idx=idx)
    torch.cuda.synchronize()
    p, j = b.slots(0)
    for g in range(2):
        w = W0[p.clamp(min=0), g, j].cpu()
        w[48:64] = float("nan")
        kept = evict_plain(w, 200, 100, 0, 0)
        assert torch.equal(idx[0, g].cpu().long(), kept)
        t = [i for i in range(100) if not 48 <= i < 64]
        got = b.K[p[t], g, j[t]]
        assert torch.equal(got, K0[p[kept[t]], g, j[kept[t]]])


# ---- all together ----

@pytest.mark.parametrize("dtype", [F32, BF16])
def test_a_generation(dtype):
    """Prompts in chunks, tokens one by one, a cut in between: every step against a cache of lists on the CPU."""
    H_q, H_kv, D, page, n_s, keep = 4, 2, 64, 16, 3, 48
    G = H_q // H_kv
    gen = torch.Generator().manual_seed(9)
    pages_each = 12
    pool = n_s * pages_each
    K = torch.full((pool, H_kv, page, D), float("nan"), dtype=dtype, device="cuda")
    V, W = K.clone(), torch.full((pool, H_kv, page), float("nan"), device="cuda")
    table = torch.randperm(pool, generator=gen).to(torch.int32).view(n_s, pages_each).cuda()
    kv = torch.zeros(n_s, dtype=torch.int32, device="cuda")
    cache = [[(torch.zeros((0, D), dtype=dtype), torch.zeros((0, D), dtype=dtype), torch.zeros(0, dtype=torch.float64),
               torch.zeros(0, dtype=torch.float64)) for _ in range(H_kv)] for _ in range(n_s)]
    steps = [(60, 7, 90), (20, 0, 33), (1, 1, 1), "evict", (1, 1, 1), (5, 0, 2), "evict", (1, 1, 1)]
    for step in steps:
        if step == "evict":
            p = dhsa.paged_problem(K, V, table, H_q, 0)
            idx = torch.zeros((n_s, H_kv, keep), dtype=torch.int32, device="cuda")
            dhsa.dhsa_paged_evict(p, K, V, W, table, kv, keep, 2, 8, dhsa.alloc_evict(p, keep), kv, idx=idx)
            torch.cuda.synchronize()
            for s in range(n_s):
                for g in range(H_kv):
                    kc, vc, wc, tc = cache[s][g]
                    kept = idx[s, g][idx[s, g] >= 0].cpu().long()
                    assert len(kept) == min(len(kc), keep) == int(kv[s])
                    if len(kc) > keep:     # what stayed is heaviest, as far as the sums are exact
                        middle = torch.zeros(len(kc), dtype=torch.bool)
                        middle[2:len(kc) - 8] = True
                        gone = middle.clone()
                        gone[kept] = False
                        stay = middle & ~gone
                        assert bool(stay[:2].any()) is False
                        assert (wc[stay] + tc[stay]).min() >= (wc[gone] - tc[gone]).max()
                    cache[s][g] = (kc[kept], vc[kept], wc[kept], tc[kept])
            continue
        T = sum(step)
        Q = torch.randn((H_q, T, D), generator=gen).to(dtype).cuda()
        Kn, Vn = (torch.randn((H_kv, T, D), generator=gen).to(dtype).cuda() for _ in range(2))
        starts = [0]
        for n in step:
            starts.append(starts[-1] + n)
        kv += torch.tensor(step, dtype=torch.int32).cuda()
        q_start = torch.tensor(starts, dtype=torch.int32).cuda()
        p = dhsa.paged_problem(K, V, table, H_q, T)
        O, lse = torch.empty_like(Q), torch.empty((H_q, T), device="cuda")
        dhsa.dhsa_paged_append(p, Kn, Vn, K, V, table, q_start, kv, W)
        dhsa.dhsa_paged_attend(p, Q, K, V, table, q_start, kv, O, dhsa.alloc_paged(p), lse=lse, weights=W, decay=0.75)
        torch.cuda.synchronize()
        for s, n in enumerate(step):
            rows = slice(starts[s], starts[s + 1])
            for g in range(H_kv):
                kc, vc, wc, tc = cache[s][g]
                kc, vc = torch.cat([kc, Kn[g, rows].cpu()]), torch.cat([vc, Vn[g, rows].cpu()])
                wc, tc = (torch.cat([x, torch.zeros(n, dtype=torch.float64)]) for x in (wc, tc))
                m = len(kc)
                assert m == int(kv[s])
                if n:
                    o, z, got, t_o, t_z, t_w = paged_plain.attend(Q[g * G:(g + 1) * G, rows].cpu(), kc, vc, torch.arange(m - n, m), 0, 0)
                    paged_plain.close(O[g * G:(g + 1) * G, rows], o, t_o, f"{step} {s} {g}")
                    paged_plain.close(lse[g * G:(g + 1) * G, rows], z, t_z, f"{step} {s} {g}")
                else:
                    got = t_w = torch.zeros(m, dtype=torch.float64)
                wc, tc = 0.75 * wc + got, 0.75 * tc + t_w + 2.0 ** -23 * (0.75 * wc + got)
                j = torch.arange(m)
                paged_plain.close(W[table[s].cpu().long()[j // page], g, j % page], wc, tc, f"weights {step} {s} {g}")
                cache[s][g] = (kc, vc, wc, tc)


def test_captured_and_replayed():
    """Append, attend and evict in one graph; lengths, pages and tokens change between the replays, and eager calls come in
    between that share its workspaces."""
    a = Batch([(1, 500), (1, 500), (2, 500)], 4, 2, 64, BF16, 16, seed=3, spare=80)     # (every sequence has its own 32 pages)
    a.K.nan_to_num_(0.0); a.V.nan_to_num_(0.0)
    keep = 64
    out_table = torch.zeros_like(a.table)
    free = [i for i in range(a.K.shape[0]) if i not in set(int(x) for x in a.table.flatten())]
    for s in range(3):
        for i in range(4):
            out_table[s, i] = free.pop()
    Kn, Vn = (torch.randn((2, a.T, 64), device="cuda").to(BF16) for _ in range(2))
    W = torch.rand((a.K.shape[0], 2, 16), device="cuda")
    O, lse, ws, wse = torch.empty_like(a.Q), torch.empty((4, a.T), device="cuda"), dhsa.alloc_paged(a.prob), dhsa.alloc_evict(a.prob, keep)
    kv_out, idx = torch.empty_like(a.kv_len), torch.empty((3, 2, keep), dtype=torch.int32, device="cuda")

    def calls():
        dhsa.dhsa_paged_append(a.prob, Kn, Vn, a.K, a.V, a.table, a.q_start, a.kv_len, W)
        dhsa.dhsa_paged_attend(a.prob, a.Q, a.K, a.V, a.table, a.q_start, a.kv_len, O, ws, lse=lse, weights=W, decay=0.5)
        dhsa.dhsa_paged_evict(a.prob, a.K, a.V, W, a.table, a.kv_len, keep, 2, 9, wse, kv_out, table_out=out_table, idx=idx)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        calls()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    for lens, starts in (((200, 77, 500), (0, 1, 2, 4)), ((33, 70, 480), (0, 2, 2, 3)), ((1, 79, 100), (0, 0, 4, 4)), ((200, 77, 500), (0, 1, 2, 4))):
        a.kv_len.copy_(torch.tensor(lens, dtype=torch.int32))
        a.q_start.copy_(torch.tensor(starts, dtype=torch.int32))
        a.table.copy_(a.table.roll(1, 0) if lens[0] == 33 else a.table)
        a.Q.copy_(torch.randn(a.Q.shape, device="cuda").to(BF16))
        Kn.copy_(torch.randn(Kn.shape, device="cuda").to(BF16))
        state = [x.clone() for x in (a.K, a.V, W)]
        for x in (O, lse):
            x.fill_(3.0)
        graph.replay()
        torch.cuda.synchronize()
        got = [x.clone() for x in (O, lse, a.K, a.V, W, kv_out, idx)]
        for x, y in zip((a.K, a.V, W), state):
            x.copy_(y)
        for x in (O, lse):
            x.fill_(3.0)
        calls()
        torch.cuda.synchronize()
        for x, y in zip(got, (O, lse, a.K, a.V, W, kv_out, idx)):
            assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))


def test_two_graphs_share_a_workspace():
    """Two captured calls of different lengths over one workspace, replayed in turn, eager calls in between."""
    a, b = Batch([(1, 3000), (1, 50)], 4, 2, 64, BF16, 16, seed=1), Batch([(1, 20), (1, 4000)], 4, 2, 64, BF16, 16, seed=2)
    ws = torch.empty(max(dhsa.dhsa_paged_workspace_bytes(x.prob) for x in (a, b)), dtype=torch.uint8, device="cuda")
    graphs = []
    for x in (a, b):
        O, lse, W = torch.empty_like(x.Q), torch.empty((4, x.T), device="cuda"), x.new_weights()
        before = W.clone()

        def call(x=x, O=O, lse=lse, W=W):
            dhsa.dhsa_paged_attend(x.prob, x.Q, x.K, x.V, x.table, x.q_start, x.kv_len, O, ws, lse=lse, weights=W, decay=0.0)

        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            call()
        torch.cuda.current_stream().wait_stream(side)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call()
        graphs.append((x, O, lse, W, before, graph, call))
    for turn in range(3):
        for x, O, lse, W, before, graph, call in graphs:
            for y in (O, lse):
                y.fill_(7.0)
            graph.replay()
            if turn == 1:
                call()
        torch.cuda.synchronize()
        for x, O, lse, W, before, graph, call in graphs:
            x.check(O, lse, before, W, 0.0)


def test_refusals_on_the_device():
    b = Batch([(1, 20), (2, 30)], 4, 2, 64, BF16, 16)
    ws, O = dhsa.alloc_paged(b.prob, weights=False), torch.empty_like(b.Q)
    good = dict(Q=b.Q, K=b.K, V=b.V, table=b.table, q_start=b.q_start, kv_len=b.kv_len, O=O, lse=None, weights=None)
    W = b.new_weights()
    for bad in (dict(Q=b.Q[:, :2]), dict(Q=b.Q.float()), dict(K=b.K[:-1]), dict(K=b.K.permute(0, 2, 1, 3)), dict(table=b.table.long()),
                dict(table=b.table[:, :1]), dict(q_start=b.q_start[:-1]), dict(kv_len=b.kv_len.float()), dict(O=O.float()),
                dict(lse=torch.empty((4, 4), device="cuda")), dict(weights=W.double()), dict(weights=W[:, :1]),
                dict(weights=W.permute(0, 2, 1).contiguous().permute(0, 2, 1))):
        t = dict(good)
        t.update(bad)
        with pytest.raises(ValueError):
            dhsa.dhsa_paged_attend(b.prob, t["Q"], t["K"], t["V"], t["table"], t["q_start"], t["kv_len"], t["O"], ws, lse=t["lse"],
                                   weights=t["weights"])
    with pytest.raises(dhsa.DhsaError) as e:
        dhsa.dhsa_paged_attend(b.prob, b.Q, b.K, b.V, b.table, b.q_start, b.kv_len, O, ws[:-1])
    assert e.value.code == 6
    with pytest.raises(ValueError):
        dhsa.dhsa_paged_evict(b.prob, b.K, b.V, W, b.table, b.kv_len, 8, 0, 0, ws, b.kv_len, idx=torch.empty((2, 2, 9), dtype=torch.int32,
                                                                                                         device="cuda"))
    with pytest.raises(dhsa.DhsaError) as e:
        dhsa.dhsa_paged_evict(b.prob, b.K, b.V, W, b.table, b.kv_len, 8, 5, 4, ws, b.kv_len)
    assert e.value.code == 4
