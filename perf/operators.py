"""Attention of a serving loop over a cache that is paged, windowed or cut down, as cases that can be timed and compared.

Each case names one operator and a problem:

  window   attention of a prompt in which a row sees the last `window` keys and the first `sinks` (dhsa_window_prefill)
  attend   attention of new tokens, one or many a sequence, over a paged cache, with the window or without; where `weights` is
           set also what each cached key got of it, summed over the rows and heads that read it (dhsa_paged_attend)
  append   the keys and values of new tokens written into the pages of their sequences (dhsa_paged_append)
  evict    all but `keep` tokens of each sequence and kv-head dropped, by what they got (dhsa_paged_evict)

Head counts, lengths and budgets are those of the configurations of dhsa_inputs.  Where `own` is false, run() computes the same in
elementary torch operations.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def _window(L, H_q, H_kv, D, dtype, window, sinks, layout="hld"):
    return dict(op="window", L=L, H_q=H_q, H_kv=H_kv, D=D, dtype=dtype, window=window, sinks=sinks, layout=layout)


def _paged(op, n_seq, q_lo, q_hi, kv_lo, kv_hi, H_q, H_kv, D, dtype, page, **options):
    """n_seq sequences of q_lo..q_hi new tokens; each has kv_lo..kv_hi tokens with them, drawn from the logarithm's range."""
    c = dict(op=op, n_seq=n_seq, q_lo=q_lo, q_hi=q_hi, kv_lo=kv_lo, kv_hi=kv_hi, H_q=H_q, H_kv=H_kv, D=D, dtype=dtype, page=page,
             window=0, sinks=0, weights=False, layout="hld", keep=0, first=0, recent=0, lengths=1)
    c.update(options)
    return c


def listed():
    cases = {
        # a short fp32 prompt of odd length: launches and latency count
        "window_short_f32": _window(1021, 4, 1, 64, "f32", 256, 4),
        # an ordinary prompt, 32K tokens, projections as a model has them ([L, H, D] rows)
        "window_32k": _window(32768, 32, 8, 128, "bf16", 2048, 4, layout="lhd"),
        # the longest prompt, as many keys a row as the headline budget of 128K tokens
        "window_128k": _window(131072, 32, 8, 128, "bf16", 8192, 64),
        # a handful of short conversations, a token each: the smallest step of a serving loop
        "attend_few_f32": _paged("attend", 4, 1, 1, 100, 1000, 8, 2, 64, "f32", 16),
        # a full batch of conversations, a token each, with the bookkeeping that eviction lives on
        "attend_batch": _paged("attend", 64, 1, 1, 1000, 32768, 32, 8, 128, "bf16", 64, weights=True),
        # one conversation at full context
        "attend_long": _paged("attend", 1, 1, 1, 131072, 131072, 32, 8, 128, "bf16", 64),
        # a prompt that is prefilled in chunks: 2048 new tokens behind 30K
        "attend_chunk": _paged("attend", 1, 2048, 2048, 32768, 32768, 32, 8, 128, "bf16", 64),
        # prompts in chunks and short turns in one batch, groups of seven heads, small pages, window and bookkeeping
        "attend_ragged": _paged("attend", 12, 1, 1024, 1500, 20000, 28, 4, 128, "bf16", 16, window=4096, sinks=4, weights=True,
                                layout="lhd"),
        # the new tokens of a batch's step go into their pages
        "append_step": _paged("append", 64, 1, 1, 1000, 8192, 32, 8, 128, "bf16", 64),
        # ... and those of prompts
        "append_prompts": _paged("append", 8, 500, 4000, 4000, 8192, 32, 8, 128, "bf16", 16, layout="lhd"),
        # a small cache is cut down between turns
        "evict_few": _paged("evict", 3, 0, 0, 900, 3000, 8, 2, 64, "bf16", 16, keep=256, first=4, recent=64),
        # prompts of up to 32K tokens are cut to an eighth after they have been read
        "evict_prompts": _paged("evict", 8, 0, 0, 8192, 32768, 32, 8, 128, "bf16", 64, keep=4096, first=4, recent=1024),
    }
    return [dict(c, name=n) for n, c in cases.items()]


def _log(rng, lo, hi):
    """A whole number between lo and hi, spread over the logarithm."""
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["window", "attend", "attend", "append", "evict"])
    H_q, H_kv = rng.choice([(4, 1), (8, 2), (32, 8), (28, 4), (16, 16)])
    D, dtype, layout = rng.choice([64, 128]), rng.choice(["bf16", "bf16", "f32"]), rng.choice(["hld", "lhd"])
    if op == "window":
        return _window(_log(rng, 1, 65536 if dtype == "bf16" else 12000), H_q, H_kv, D, dtype,
                       _log(rng, 1, 8192 if dtype == "bf16" else 2048), rng.choice([0, 1, 4, 64, 333]), layout)
    page = rng.choice([1, 16, 16, 24, 64, 64, 256])
    n_seq = _log(rng, 1, 64)
    kv_hi = _log(rng, 1, min(131072, (1 << 21) // n_seq * 8 // H_kv // (1 if dtype == "bf16" else 2)))
    kv_lo = _log(rng, 1, kv_hi)
    lengths = rng.randrange(1 << 30)
    if op == "evict":
        keep = _log(rng, 1, max(1, kv_hi))
        first = rng.randint(0, min(8, keep))
        return _paged(op, n_seq, 0, 0, kv_lo, kv_hi, H_q, H_kv, D, dtype, page, keep=keep, first=first,
                      recent=rng.randint(0, keep - first), lengths=lengths)
    q_hi = rng.choice([1, 1, _log(rng, 1, 8), _log(rng, 1, max(1, min(kv_hi, 4096 // n_seq)))])
    q_lo = rng.randint(0 if q_hi > 1 else 1, q_hi)
    window = rng.choice([0, 0, _log(rng, 1, max(1, kv_hi))]) if op == "attend" else 0
    return _paged(op, n_seq, q_lo, q_hi, kv_lo, kv_hi, H_q, H_kv, D, dtype, page, window=window,
                  sinks=rng.choice([0, 4, 100]) if window else 0, weights=op == "attend" and rng.random() < 0.4, layout=layout,
                  lengths=lengths)


def _lengths(case):
    """(new tokens, tokens with them) of each sequence; the first has the most of both."""
    rng = random.Random(case["lengths"])
    out = []
    for s in range(case["n_seq"]):
        kv = case["kv_hi"] if s == 0 else _log(rng, case["kv_lo"], case["kv_hi"])
        q = case["q_hi"] if s == 0 else case["q_lo"] if case["q_lo"] == case["q_hi"] else rng.randint(case["q_lo"], case["q_hi"])
        out.append((min(q, kv), kv))
    return out


def _loud(gen, x):
    """One key in a hundred four times as loud, so that attention has something to find."""
    loud = torch.rand(x.shape[:-1], generator=gen, device="cuda") < 0.01
    return x * torch.where(loud, 4.0, 1.0)[..., None].to(x.dtype)


def _rows(gen, heads, n, D, dt, layout, loud=False):
    """[heads, n, D], in memory as it says or as [n, heads, D]."""
    x = torch.randn((heads, n, D) if layout == "hld" else (n, heads, D), generator=gen, device="cuda", dtype=torch.float32)
    if loud:
        x = _loud(gen, x)
    x = x.to(dt)
    return x if layout == "hld" else x.permute(1, 0, 2)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    dt = DTYPES[case["dtype"]]
    H_q, H_kv, D = case["H_q"], case["H_kv"], case["D"]
    s = dict(case=case)
    if own:
        import paper_2510_24606_amd as dhsa
        s["dhsa"] = dhsa
    if case["op"] == "window":
        L = case["L"]
        s["Q"], s["V"] = _rows(gen, H_q, L, D, dt, case["layout"]), _rows(gen, H_kv, L, D, dt, case["layout"])
        s["K"] = _rows(gen, H_kv, L, D, dt, case["layout"], loud=True)
        s["O"] = torch.empty_like(s["Q"])
        if own:
            s["prob"] = dhsa.problem(s["Q"], s["K"], [0, L], L, V=s["V"])
        return s
    lens = _lengths(case)
    page, n_seq = case["page"], case["n_seq"]
    T = sum(q for q, _ in lens)
    need = [-(-kv // page) for _, kv in lens]
    kept = [-(-min(kv, case["keep"]) // page) for _, kv in lens] if case["op"] == "evict" else [0] * n_seq
    n_pages, widest = sum(need) + sum(kept) + 3, max(need)
    # the pool: pages in any order; what no token has been written to is left as it was
    K = torch.randn((n_pages, H_kv, page, D), generator=gen, device="cuda").to(dt)
    s["K"] = _loud(gen, K) if case["op"] == "attend" else K
    s["V"] = torch.randn((n_pages, H_kv, page, D), generator=gen, device="cuda").to(dt)
    order = torch.randperm(n_pages, generator=gen, device="cuda").to(torch.int32)
    at = [0]
    for n in need + kept:
        at.append(at[-1] + n)
    table = torch.zeros((n_seq, widest), dtype=torch.int32, device="cuda")
    table_out = torch.zeros((n_seq, widest), dtype=torch.int32, device="cuda")
    for i in range(n_seq):
        table[i, :need[i]] = order[at[i]:at[i + 1]]
        table_out[i, :kept[i]] = order[at[n_seq + i]:at[n_seq + i + 1]]
    starts = [0]
    for q, _ in lens:
        starts.append(starts[-1] + q)
    s.update(table=table, lens=lens, starts=starts, T=T, kv_len=torch.tensor([kv for _, kv in lens], dtype=torch.int32, device="cuda"),
             q_start=torch.tensor(starts, dtype=torch.int32, device="cuda"), lse=None, W=None)
    if case["weights"] or case["op"] == "evict":
        # what a key has got so far: few have most of it
        s["W"] = torch.randn((n_pages, H_kv, page), generator=gen, device="cuda").mul_(2.0).exp_().mul_(1.0 if case["op"] == "evict" else 1e-6)
    if case["op"] == "attend":
        s["Q"] = _rows(gen, H_q, T, D, dt, case["layout"])
        s["O"] = torch.empty_like(s["Q"])
        s["lse"] = torch.empty((H_q, T), dtype=torch.float32, device="cuda")
    if case["op"] == "append":
        s["K_new"], s["V_new"] = _rows(gen, H_kv, T, D, dt, case["layout"]), _rows(gen, H_kv, T, D, dt, case["layout"])
    if case["op"] == "evict":
        s["table_out"], s["kv_out"] = table_out, torch.empty_like(s["kv_len"])
        s["idx"] = torch.empty((n_seq, H_kv, case["keep"]), dtype=torch.int32, device="cuda")
    if own:
        s["prob"] = dhsa.paged_problem(s["K"], s["V"], table, H_q, T, window=case["window"], sinks=case["sinks"])
        s["ws"] = dhsa.alloc_evict(s["prob"], case["keep"]) if case["op"] == "evict" else dhsa.alloc_paged(s["prob"])
    return s


# ---- the plain forms ----

BLOCK = 1 << 28     # scores that are held at a time


def _attend(q, k, v, pos, at, window, sinks, scale):
    """Rows q [H_kv, G, n, D] at the positions pos [n], keys and values [H_kv, m, D] at the positions at [m], all fp32:
    (output, log of the sum of exponentials [H_kv, G, n], what each key got [H_kv, m])."""
    H_kv, G, n, D = q.shape
    sees = at[None, :] <= pos[:, None]
    if window > 0:
        sees &= (pos[:, None] - at[None, :] < window) | (at[None, :] < sinks)
    x = torch.matmul(q.reshape(H_kv, G * n, D), k.transpose(1, 2).contiguous()).mul_(scale).view(H_kv, G, n, -1)
    x.masked_fill_(~sees, -math.inf)
    top = x.amax(-1, keepdim=True)
    x.sub_(top).exp_()
    total = x.sum(-1, keepdim=True)
    x.div_(total)
    o = torch.matmul(x.view(H_kv, G * n, -1), v).view(H_kv, G, n, D)
    return o, (top + total.log()).squeeze(-1), x.sum((1, 2))


def _run_window(s):
    c = s["case"]
    L, H_q, H_kv, D = c["L"], c["H_q"], c["H_kv"], c["D"]
    G, window, sinks = H_q // H_kv, c["window"], c["sinks"]
    step = max(1, min(L, 2048, BLOCK // (H_q * (window + sinks + 2048))))
    pos = torch.arange(L, device="cuda")
    for i in range(0, L, step):
        j = min(i + step, L)
        lo = max(0, i - window + 1)
        keep = min(sinks, lo)
        at = torch.cat([pos[:keep], pos[lo:j]])
        k = torch.cat([s["K"][:, :keep], s["K"][:, lo:j]], 1).float()
        v = torch.cat([s["V"][:, :keep], s["V"][:, lo:j]], 1).float()
        q = s["Q"][:, i:j].float().reshape(H_kv, G, j - i, D)
        s["O"][:, i:j] = _attend(q, k, v, pos[i:j], at, window, sinks, D ** -0.5)[0].reshape(H_q, j - i, D).to(s["O"].dtype)
    return s["O"]


def _slots(s, i, n):
    """(page, slot) of the first n tokens of sequence i."""
    page = s["case"]["page"]
    at = torch.arange(n, device="cuda")
    return s["table"][i].long()[at // page], at % page


def _run_attend(s):
    c = s["case"]
    H_q, H_kv, D = c["H_q"], c["H_kv"], c["D"]
    G, window, sinks = H_q // H_kv, c["window"], c["sinks"]
    for i, (n, kv) in enumerate(s["lens"]):
        page, slot = _slots(s, i, kv)
        k, v = s["K"][page, :, slot].float().transpose(0, 1), s["V"][page, :, slot].float().transpose(0, 1)
        at, got = torch.arange(kv, device="cuda"), torch.zeros((H_kv, kv), device="cuda")
        step = max(1, BLOCK // (H_q * kv))
        for a in range(0, n, step):
            b = min(a + step, n)
            rows = slice(s["starts"][i] + a, s["starts"][i] + b)
            first = kv - n + a
            lo = max(0, first - window + 1) if window > 0 else 0
            keep = min(sinks, lo)
            some = torch.cat([at[:keep], at[lo:kv - n + b]])
            q = s["Q"][:, rows].float().reshape(H_kv, G, b - a, D)
            o, lse, w = _attend(q, k[:, some], v[:, some], at[kv - n + a:kv - n + b], some, window, sinks, D ** -0.5)
            s["O"][:, rows] = o.reshape(H_q, b - a, D).to(s["O"].dtype)
            s["lse"][:, rows] = lse.reshape(H_q, b - a)
            if c["weights"]:
                got[:, some] += w
        if c["weights"]:
            s["W"][page, :, slot] = got.transpose(0, 1)
    return {"O": s["O"], "lse": s["lse"], "weights": s["W"]}


def _run_append(s):
    page, T = s["case"]["page"], s["T"]
    n = s["q_start"][1:] - s["q_start"][:-1]
    seq = torch.repeat_interleave(torch.arange(len(n), device="cuda"), n, output_size=T)
    at = torch.arange(T, device="cuda") - s["q_start"][seq] + (s["kv_len"] - n)[seq]
    to_page, to_slot = s["table"][seq, at // page].long(), at % page
    s["K"][to_page, :, to_slot] = s["K_new"].transpose(0, 1)
    s["V"][to_page, :, to_slot] = s["V_new"].transpose(0, 1)
    return {"K": s["K"], "V": s["V"]}


def _run_evict(s):
    c = s["case"]
    page, keep = c["page"], c["keep"]
    n_seq, H_kv, most = c["n_seq"], c["H_kv"], max(kv for _, kv in s["lens"])
    kv = s["kv_len"].long()[:, None, None]
    at = torch.arange(most, device="cuda")
    head = torch.arange(H_kv, device="cuda")[None, :, None]
    w = s["W"][s["table"].long()[:, None, at // page], head, at % page]                     # [n_seq, H_kv, most]
    w = torch.where((at < c["first"]) | (at >= kv - c["recent"]), math.inf, w).masked_fill_(at >= kv, -math.inf)
    rank = torch.sort(w, dim=-1, descending=True, stable=True)[1][..., :keep]
    rank = torch.nn.functional.pad(rank, (0, keep - rank.shape[-1]), value=most)
    kept = torch.sort(rank.masked_fill(rank >= kv, most), dim=-1)[0]
    there = kept < most
    s["idx"].copy_(kept.masked_fill(~there, -1))
    seq, head, to = torch.nonzero(there, as_tuple=True)
    at = kept[seq, head, to]
    from_page, to_page = s["table"][seq, at // page].long(), s["table_out"][seq, to // page].long()
    for x in (s["K"], s["V"], s["W"]):
        x[to_page, head, to % page] = x[from_page, head, at % page]
    s["kv_out"].copy_(torch.clamp(s["kv_len"], max=keep))
    return {"K": s["K"], "V": s["V"], "weights": s["W"], "kv_len": s["kv_out"], "idx": s["idx"]}


def run(state):
    s = state
    c = s["case"]
    if own:
        dhsa = s["dhsa"]
        if c["op"] == "window":
            dhsa.dhsa_window_prefill(s["prob"], s["Q"], s["K"], s["V"], s["O"], c["window"], c["sinks"])
            return s["O"]
        if c["op"] == "attend":
            # decay 0: the weights of this call alone
            dhsa.dhsa_paged_attend(s["prob"], s["Q"], s["K"], s["V"], s["table"], s["q_start"], s["kv_len"], s["O"], s["ws"],
                                   lse=s["lse"], weights=s["W"], decay=0.0)
            return {"O": s["O"], "lse": s["lse"], "weights": s["W"]}
        if c["op"] == "append":
            dhsa.dhsa_paged_append(s["prob"], s["K_new"], s["V_new"], s["K"], s["V"], s["table"], s["q_start"], s["kv_len"])
            return {"K": s["K"], "V": s["V"]}
        dhsa.dhsa_paged_evict(s["prob"], s["K"], s["V"], s["W"], s["table"], s["kv_len"], c["keep"], c["first"], c["recent"],
                              s["ws"], s["kv_out"], table_out=s["table_out"], idx=s["idx"])
        return {"K": s["K"], "V": s["V"], "weights": s["W"], "kv_len": s["kv_out"], "idx": s["idx"]}
    return {"window": _run_window, "attend": _run_attend, "append": _run_append, "evict": _run_evict}[c["op"]](s)


# ---- the definition in 64 bits ----

def _exact_rows(Q, K, V, pos, window, sinks, scale):
    """One kv-head: Q [G, n, D] at pos [n], K and V [m, D] at 0..m-1, row by row in blocks: (output, log-sum, sum over rows of the weights)."""
    G, n, D = Q.shape
    out, lse, got = torch.zeros_like(Q), torch.zeros((G, n), dtype=Q.dtype, device="cuda"), torch.zeros(K.shape[0], dtype=Q.dtype, device="cuda")
    block = max(1, min(1024, (1 << 26) // (K.shape[0] if window == 0 else min(K.shape[0], window + 1024))))
    for a in range(0, n, block):
        p = pos[a:a + block]
        lo = 0 if window == 0 else max(0, int(p[0]) - window + 1)
        j = torch.arange(int(p[-1]) + 1, device="cuda")
        j = torch.cat([j[:min(sinks, lo)], j[lo:]])
        distance = p[:, None] - j[None, :]
        visible = distance >= 0
        if window:
            visible = visible & ((distance < window) | (j < sinks)[None, :])
        for g in range(G):
            logits = Q[g, a:a + block] @ K[j].T * scale
            logits = torch.where(visible, logits, torch.full_like(logits, -math.inf))
            m = logits.max(1, keepdim=True).values
            e = torch.exp(logits - m)
            z = e.sum(1, keepdim=True)
            out[g, a:a + block] = (e @ V[j]) / z
            lse[g, a:a + block] = (m + torch.log(z))[:, 0]
            got[j] += (e / z).sum(0)
    return out, lse, got


def exact(case, seed):
    s = prepare(case, seed)
    H_q, H_kv, D = case["H_q"], case["H_kv"], case["D"]
    G, scale = H_q // H_kv, 1.0 / math.sqrt(D)
    if case["op"] == "window":
        out = torch.zeros(s["Q"].shape, dtype=torch.float64, device="cuda")
        pos = torch.arange(case["L"], device="cuda")
        for g in range(H_kv):
            out[g * G:(g + 1) * G] = _exact_rows(s["Q"][g * G:(g + 1) * G].double(), s["K"][g].double(), s["V"][g].double(), pos,
                                                 case["window"], case["sinks"], scale)[0]
        return out
    page, table = case["page"], s["table"].tolist()
    if case["op"] == "attend":
        out = torch.zeros(s["Q"].shape, dtype=torch.float64, device="cuda")
        lse = torch.zeros(s["lse"].shape, dtype=torch.float64, device="cuda")
        weights = s["W"].double() if case["weights"] else None
        for i, (n, kv) in enumerate(s["lens"]):
            if n == 0 and weights is None:
                continue
            pages = torch.tensor(table[i][:-(-kv // page)], device="cuda")
            t0, t1 = s["starts"][i], s["starts"][i + 1]
            for g in range(H_kv):
                K, V = (x[pages, g].reshape(-1, D)[:kv].double() for x in (s["K"], s["V"]))
                o, z, got = _exact_rows(s["Q"][g * G:(g + 1) * G, t0:t1].double(), K, V, torch.arange(kv - n, kv, device="cuda"),
                                        case["window"], case["sinks"], scale)
                out[g * G:(g + 1) * G, t0:t1], lse[g * G:(g + 1) * G, t0:t1] = o, z
                if weights is not None:
                    whole = weights[pages, g].reshape(-1)
                    whole[:kv] = got
                    weights[pages, g] = whole.view(-1, page)
        return {"O": out, "lse": lse, "weights": weights}
    # moved values are the values themselves: nothing is computed that 64 bits would do better
    return None


# ---- what a pass cannot do without ----

def _pairs(n, kv, window, sinks):
    """(row, key) pairs that n rows at the end of kv tokens see, and the keys that any of them sees."""
    pairs = n * (kv - n) + n * (n + 1) // 2
    if n == 0:
        return 0, 0
    if window <= 0:
        return pairs, kv
    # rows at p see min(p + 1, window) of the last and min(sinks, p + 1 - window) of the first
    def upto(p, most):      # sum over q = 0 .. p-1 of min(q + 1, most)
        m = min(p, most)
        return m * (m + 1) // 2 + (p - m) * most
    seen = upto(kv, window) - upto(kv - n, window)
    a, b = max(0, kv - window), max(0, kv - n - window)
    seen += upto(a, sinks) - upto(b, sinks)
    lo = max(0, kv - n - window + 1)
    return seen, min(sinks, lo) + kv - lo


def work(case):
    H_q, H_kv, D = case["H_q"], case["H_kv"], case["D"]
    size = 4.0 if case["dtype"] == "f32" else 2.0
    if case["op"] == "window":
        pairs, _ = _pairs(case["L"], case["L"], case["window"], case["sinks"])
        return {"bytes": (2.0 * H_q + 2.0 * H_kv) * case["L"] * D * size, "flops": 4.0 * D * H_q * pairs}
    total = {"bytes": 0.0, "flops": 0.0}
    for n, kv in _lengths(case):
        total["bytes"] += 4.0 * -(-kv // case["page"]) + 8.0
        if case["op"] == "attend":
            pairs, keys = _pairs(n, kv, case["window"], case["sinks"])
            total["bytes"] += 2.0 * H_kv * keys * D * size + 2.0 * H_q * n * D * size + 4.0 * H_q * n
            total["bytes"] += 4.0 * H_kv * kv if case["weights"] else 0.0
            total["flops"] += 4.0 * D * H_q * pairs + (H_q * pairs if case["weights"] else 0.0)
        elif case["op"] == "append":
            total["bytes"] += 4.0 * H_kv * n * D * size
        else:
            m = min(kv, case["keep"])
            total["bytes"] += 4.0 * H_kv * kv + 4.0 * H_kv * m * D * size + 8.0 * H_kv * m
    return total
