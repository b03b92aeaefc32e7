"""Rotary positions, the cache in pages and the attention of one new token over it, against the fp64 oracle.

Bounds.  A turned element is x cos - y sin with sine and cosine of fp32 (2^-22 off: the angle's fraction of a turn is rounded to fp32 once; and
|angle| 2^-50: a few roundings of 64 bits here and in the oracle) in two fp32 steps, rounded once to bf16:
(2^-22 + 2^-23 + |angle| 2^-50) (|x| + |y|) amplitude + h |want|, h = 2^-8.  Attention as in test_gpu_attention.py;
parts are joined in fp32, each with a factor of its own: 2^-22 more."""
import numpy as np
import pytest
import torch

from oracle import attention as A
from paper_2407_08296_amd import qgalore as qg

pytestmark = pytest.mark.gpu
DEV = "cuda"
H = 2.0 ** -8
np64 = lambda t: t.detach().float().cpu().numpy().astype(np.float64)


def normal(*shape, seed=0, std=1.0):
    return (torch.randn(*shape, generator=torch.Generator().manual_seed(seed)) * std).bfloat16().to(DEV)


def turned(x, got, pos, freqs, layout, amplitude=1.0, backward=False):
    """got is x turned, within the bound."""
    X = np64(x)
    want = A.rope(X, pos.tolist(), freqs.cpu().numpy(), layout, amplitude, backward)
    half = len(freqs)
    size = np.zeros_like(X)
    first, second = (slice(0, half), slice(half, 2 * half)) if layout == "half" else (slice(0, 2 * half, 2), slice(1, 2 * half, 2))
    size[..., first] = size[..., second] = np.abs(X[..., first]) + np.abs(X[..., second])
    angle = np.abs(pos.cpu().numpy().astype(np.float64))[:, None, None] * float(freqs.max()) * 2.0 ** -50
    tol = abs(amplitude) * (2.0 ** -22 + 2.0 ** -23 + angle) * size + np.where(size > 0, H, 0.0) * np.abs(want) + np.where(size > 0, 1e-38, 0.0)
    off = np.abs(np64(got) - want)
    assert np.all(off <= tol), float((off - tol).max())
    assert np.array_equal(np64(got)[..., 2 * half:], X[..., 2 * half:])


POSITIONS = [0, 1, 7, 4095, 123456, 999999, 2 ** 31 + 11]


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("tokens,heads,heads_k,d,rot", [(1, 1, 1, 8, 2), (7, 12, 12, 64, 64), (3, 4, 1, 128, 128), (5, 2, 2, 80, 20), (9, 3, 1, 96, 94), (600, 3, 1, 40, 14),
                                                        (1100, 12, 4, 64, 32), (2, 2, 0, 1024, 1024), (70, 1, 1, 16, 6), (33, 5, 5, 128, 96)])
def test_rope(tokens, heads, heads_k, d, rot, layout):
    q, k = normal(tokens, heads, d, seed=1), normal(tokens, heads_k, d, seed=2) if heads_k else None
    pos = torch.tensor([POSITIONS[i % 7] + i // 7 for i in range(tokens)], dtype=torch.int64, device=DEV)
    freqs = qg.rope_frequencies(rot, factor=8.0, context=4096)
    assert np.allclose(freqs.cpu().numpy(), A.rope_frequencies(rot, factor=8.0, context=4096), rtol=1e-14)
    for f, backward in ((qg.rope_forward, False), (qg.rope_backward, True)):
        a, b = f(q, k, pos, freqs, layout, 1.25)
        turned(q, a, pos, freqs, layout, 1.25, backward)
        if k is None:
            assert b is None
        else:
            turned(k, b, pos, freqs, layout, 1.25, backward)
    inq, ink = q.clone(), None if k is None else k.clone()
    qg.rope_forward(inq, ink, pos, freqs, layout, out=(inq, ink))
    a, b = qg.rope_forward(q, k, pos, freqs, layout)
    assert torch.equal(inq, a) and (k is None or torch.equal(ink, b))


def test_rope_of_slices_in_place():
    """q and k inside one layer's output; v beside them stays as it was."""
    x = normal(50, (4 + 2 + 2) * 64, seed=3)
    before = x.clone()
    pos, freqs = torch.arange(50, device=DEV), qg.rope_frequencies(64)
    q, k = x[:, :256].view(50, 4, 64), x[:, 256:384].view(50, 2, 64)
    qg.rope_forward(q, k, pos, freqs, out=(q, k))
    turned(before[:, :256].view(50, 4, 64), q, pos, freqs, "half")
    turned(before[:, 256:384].view(50, 2, 64), k, pos, freqs, "half")
    assert torch.equal(x[:, 384:], before[:, 384:])


def test_rope_gradient_is_the_transpose():
    """<rope(x), g> = <x, rope_backward(g)>, exactly but for the roundings of both."""
    x, g = normal(20, 3, 64, seed=4), normal(20, 3, 64, seed=5)
    pos, freqs = torch.arange(20, device=DEV) * 1000, qg.rope_frequencies(48)
    y, _ = qg.rope_forward(x, None, pos, freqs)
    gx, _ = qg.rope_backward(g, None, pos, freqs)
    a, b = float((y.double() * g.double()).sum()), float((x.double() * gx.double()).sum())
    most = H * float((y.double() * g.double()).abs().sum() + (x.double() * gx.double()).abs().sum())
    assert abs(a - b) <= most


def make_cache(pages, page, heads, d, width, sequences, seed=0):
    k, v = normal(pages, page, heads, d, seed=seed, std=1.5), normal(pages, page, heads, d, seed=seed + 1)
    table = torch.randperm(pages, generator=torch.Generator().manual_seed(seed))[:sequences * width].to(torch.int32).view(sequences, width).to(DEV)
    return k, v, table


@pytest.mark.parametrize("layout,rot", [("half", 64), ("interleaved", 40), ("half", 0)])
@pytest.mark.parametrize("page", [1, 5, 16])
def test_append(layout, rot, page):
    sequences, width, heads, heads_k, d = 4, 40 // page + 1, 6, 2, 64
    kp, vp, table = make_cache(sequences * width + 3, page, heads_k, d, width, sequences)
    table[2, 0] = -1
    table[3, 0] = sequences * width + 3                # no such page
    q, k, v = normal(9, heads, d, seed=6), normal(9, heads_k, d, seed=7), normal(9, heads_k, d, seed=8)
    seq = torch.tensor([0, 1, 2, 3, 0, 1, 9, -1, 1], dtype=torch.int32, device=DEV)
    pos = torch.tensor([0, 39, 0, 0, 17, 3, 2, 2, 10 ** 9], dtype=torch.int64, device=DEV)
    freqs = qg.rope_frequencies(rot) if rot else None
    before = kp.clone(), vp.clone()
    q_out = qg.cache_append(q, k, v, pos, kp, vp, table, sequence=seq, freqs=freqs, layout=layout)
    if rot:
        turned(q, q_out, pos, freqs, layout)
        ks, _ = qg.rope_forward(k, None, pos, freqs, layout)
    else:
        assert torch.equal(q_out, q)
        ks = k
    want_k, want_v = before
    for t in range(9):
        at = A.cache_place(table.tolist(), int(seq[t]), int(pos[t]), page, kp.shape[0])
        assert (at is None) == (t in (2, 3, 6, 7, 8))
        if at is not None:
            want_k[at], want_v[at] = ks[t], v[t]
    assert torch.equal(kp, want_k) and torch.equal(vp, want_v)


def test_append_without_q_in_place_and_of_every_sequence():
    kp, vp, table = make_cache(8, 16, 2, 64, 2, 3)
    k, v, q = normal(3, 2, 64, seed=1), normal(3, 2, 64, seed=2), normal(3, 4, 64, seed=3)
    pos, freqs = torch.tensor([5, 20, 31], device=DEV), qg.rope_frequencies(64)
    assert qg.cache_append(None, k, v, pos, kp, vp, table, freqs=freqs) is None
    want, _ = qg.rope_forward(k, None, pos, freqs)
    for t, p in enumerate(pos.tolist()):
        assert torch.equal(kp[table[t, p // 16], p % 16], want[t]) and torch.equal(vp[table[t, p // 16], p % 16], v[t])
    q2 = q.clone()
    qg.cache_append(q2, k, v, pos, kp, vp, table, freqs=freqs, out=q2)
    assert torch.equal(q2, qg.rope_forward(q, None, pos, freqs)[0])


def check_paged(q, kp, vp, table, lengths, got, scale=None, cap=0.0, slopes=None, window=0):
    Q, K, V, O = np64(q), np64(kp), np64(vp), np64(got)
    sequences, heads, d = Q.shape
    page, heads_k = kp.shape[1:3]
    scale = d ** -0.5 if scale is None else scale
    rows = table.tolist()
    for s in range(sequences):
        at, end = A.paged_rows(rows, s, int(lengths[s]), page, kp.shape[0], window)
        if not at:
            assert not O[s].any()
            continue
        where = np.array([j for j, _ in at])
        pg, rw = np.array([a[0] for _, a in at]), np.array([a[1] for _, a in at])
        for h in range(heads):
            g = h // (heads // heads_k)
            kh, vh, qh = K[pg, rw, g], V[pg, rw, g], Q[s, h]
            x = scale * (kh @ qh)
            if cap:
                x = cap * np.tanh(x / cap)
            slope = 0.0 if slopes is None else float(slopes[h])
            x = x - slope * (end - 1 - where)
            p = np.exp(x - x.max())
            p /= p.sum()
            want = p @ vh
            e = ((d + 16) * 2.0 ** -24 * scale * (np.abs(kh) @ np.abs(qh)) + cap * 2.0 ** -21 + abs(slope) * (end - 1 - where) * 2.0 ** -23).max()
            ep = e + (len(at) + 16) * 2.0 ** -24 + np.abs(x).max() * 2.0 ** -22
            tol = 1.01 * ((H + 2 * ep) * (p @ np.abs(vh)) + H * np.abs(want)) + 1e-30
            assert np.all(np.abs(O[s, h] - want) <= tol), (s, h, float((np.abs(O[s, h] - want) / tol).max()))


def run_paged(lengths, heads, heads_k, d, page, seed=0, slack=1, **how):
    width = max(-(-max(max(lengths), 1) // page), 1) + slack
    kp, vp, table = make_cache(len(lengths) * width + 2, page, heads_k, d, width, len(lengths), seed)
    q = normal(len(lengths), heads, d, seed=seed + 5, std=1.5)
    n = torch.tensor(lengths, dtype=torch.int32, device=DEV)
    # what lies behind a sequence's end, in its own last page too, may hold anything
    for s, m in enumerate(lengths):
        for j in range(m, width * page):
            kp[table[s, j // page], j % page] = float("nan")
            vp[table[s, j // page], j % page] = float("inf")
    got = qg.attention_paged(q, kp, vp, table, n, **how)
    torch.cuda.synchronize()
    check_paged(q, kp, vp, table, lengths, got, **how)


@pytest.mark.parametrize("n", [0, 1, 15, 16, 17, 31, 32, 33, 127, 129, 511, 512, 513, 2100])
def test_paged_lengths(n):
    run_paged([n], 4, 2, 64, 16, seed=n)


# (lengths, heads, heads_k, d, page): one share of a sequence, a few, many (joined by four waves per head)
SHARES = [([100], 4, 2, 64, 16), ([700, 5], 4, 2, 64, 16), ([9000], 4, 2, 64, 16), ([9000, 0, 4000], 3, 1, 128, 100), ([6000], 2, 2, 40, 7),
          ([23000], 8, 8, 64, 16), ([20000], 2, 1, 128, 32), ([70000], 4, 4, 64, 64)]      # one sequence: parts of 384; 79 and 183 shares


@pytest.mark.parametrize("lengths,heads,heads_k,d,page", SHARES)
@pytest.mark.parametrize("window", [0, 2500])
def test_paged_shares(lengths, heads, heads_k, d, page, window):
    run_paged(lengths, heads, heads_k, d, page, seed=len(lengths), slack=0, window=window)


@pytest.mark.parametrize("d", [64, 128])
def test_paged_more_parts_than_workgroups(d):
    """700 sequences, 4 key heads: two workgroups each take a long sequence's eight parts in turn; a table far wider than most need."""
    lengths = [4000 if i in (0, 350, 699) else i % 40 for i in range(700)]
    page, width = 16, 400
    pages = sum(-(-n // page) for n in lengths)
    kp, vp = normal(pages, page, 4, d, seed=1, std=1.5), normal(pages, page, 4, d, seed=2)
    ids = torch.randperm(pages, generator=torch.Generator().manual_seed(3)).tolist()
    table, at = torch.full((700, width), -1, dtype=torch.int32), 0
    for i, n in enumerate(lengths):
        for j in range(-(-n // page)):
            table[i, j], at = ids[at], at + 1
    q = normal(700, 4, d, seed=4, std=1.5)
    got = qg.attention_paged(q, kp, vp, table.to(DEV), torch.tensor(lengths, dtype=torch.int32, device=DEV))
    check_paged(q, kp, vp, table, lengths, got)


@pytest.mark.parametrize("page", [1, 3, 16, 31, 64, 100, 1000])
def test_paged_page_sizes(page):
    run_paged([700, 5, 0, 64, 333], 4, 2, 64, page, seed=page)


@pytest.mark.parametrize("heads,heads_k,d", [(1, 1, 8), (3, 3, 40), (16, 1, 64), (17, 1, 64), (40, 2, 72), (12, 4, 88), (4, 4, 104), (32, 8, 128), (8, 2, 120), (6, 6, 128)])
def test_paged_heads(heads, heads_k, d):
    run_paged([200, 33], heads, heads_k, d, 16, seed=heads)


@pytest.mark.parametrize("how", [dict(cap=6.0), dict(slopes=True), dict(window=1), dict(window=50), dict(window=600, cap=5.0, slopes=True), dict(window=10 ** 6), dict(scale=1.0)])
@pytest.mark.parametrize("d", [64, 96, 128])
def test_paged_scores(how, d):
    how = dict(how, slopes=torch.tensor([0.5, 0.1, 0.02, 0.0], device=DEV)) if how.get("slopes") else how
    run_paged([1300, 49, 50, 51, 1], 4, 2, d, 16, seed=9, **how)


def test_paged_hidden_values_and_missing_pages():
    kp, vp, table = make_cache(40, 16, 2, 64, 8, 4, 3)
    q = normal(4, 4, 64, seed=4, std=1.5)
    table[0, 1], table[1, 0], table[2] = -1, 40, 10 ** 6
    lengths = torch.tensor([100, 100, 100, 10 ** 9], dtype=torch.int32, device=DEV)      # the last: as far as the table goes
    got = qg.attention_paged(q, kp, vp, table, lengths)
    check_paged(q, kp, vp, table, lengths.tolist(), got)
    # values that the window hides may be anything
    k2, v2 = kp.clone(), vp.clone()
    for s in range(4):
        for j in range(70):
            if 0 <= int(table[s, j // 16]) < 40:
                k2[table[s, j // 16], j % 16], v2[table[s, j // 16], j % 16] = float("nan"), float("nan")
    lengths.fill_(100)
    assert torch.equal(qg.attention_paged(q, kp, vp, table, lengths, window=30), qg.attention_paged(q, k2, v2, table, lengths, window=30))
    lengths.fill_(-5)
    assert not qg.attention_paged(q, kp, vp, table, lengths).any()


def test_paged_past_32_bits():
    """Rows of the cache beyond 2^31 and 2^32 elements."""
    page, heads, d = 64, 8, 128
    pages = (1 << 32) // (page * heads * d) + 3
    kp, vp = (torch.empty(pages, page, heads, d, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    ids = [0, pages // 2, pages - 2, pages - 1]
    table = torch.tensor([ids], dtype=torch.int32, device=DEV)
    k, v = normal(256, heads, d, seed=1, std=1.5), normal(256, heads, d, seed=2)
    seq = torch.zeros(256, dtype=torch.int32, device=DEV)
    qg.cache_append(None, k, v, torch.arange(256, device=DEV), kp, vp, table, sequence=seq)
    for i, p in enumerate(ids):
        assert torch.equal(kp[p], k[64 * i:64 * i + 64]) and torch.equal(vp[p], v[64 * i:64 * i + 64])
    q = normal(1, 8, d, seed=3, std=1.5)
    got = qg.attention_paged(q, kp, vp, table, torch.tensor([250], dtype=torch.int32, device=DEV))
    small = torch.tensor([[0, 1, 2, 3]], dtype=torch.int32, device=DEV)
    want = qg.attention_paged(q, kp[ids].contiguous(), vp[ids].contiguous(), small, torch.tensor([250], dtype=torch.int32, device=DEV))
    assert torch.equal(got, want)
    check_paged(q, kp[ids], vp[ids], small, [250], want)


def test_prompt_then_tokens_one_by_one():
    """The operators as a program calls them: a prompt through rope, attention and into the cache, then token after token over the cache;
    each token's output is that of the whole sequence's attention."""
    T, first, heads, heads_k, d, page = 90, 61, 4, 2, 64, 16
    q, k, v = normal(T, heads, d, seed=1, std=1.5), normal(T, heads_k, d, seed=2, std=1.5), normal(T, heads_k, d, seed=3)
    freqs, pos = qg.rope_frequencies(d), torch.arange(T, device=DEV)
    kp, vp, table = make_cache(10, page, heads_k, d, 6, 1)
    qr, kr = qg.rope_forward(q, k, pos, freqs)
    whole, _ = qg.attention_forward(qr, kr, v, cap=9.0)
    zero = torch.zeros(T, dtype=torch.int32, device=DEV)
    qa = qg.cache_append(q[:first], k[:first], v[:first], pos[:first], kp, vp, table, sequence=zero[:first], freqs=freqs)
    assert torch.equal(qa, qr[:first])
    for t in range(first, T):
        qt = qg.cache_append(q[t:t + 1], k[t:t + 1], v[t:t + 1], pos[t:t + 1], kp, vp, table, freqs=freqs)
        n = torch.tensor([t + 1], dtype=torch.int32, device=DEV)
        got = qg.attention_paged(qt, kp, vp, table, n, cap=9.0)
        check_paged(qt, kp, vp, table, [t + 1], got, cap=9.0)
        # both are within h (sum p |v| + |o|) of the exact value
        assert float((got[0].double() - whole[t].double()).abs().max()) <= 4 * H * float(v.double().abs().max())


def test_decoding_captured_in_two_graphs():
    """A step captured once and replayed as the sequences grow; a second graph has a workspace of its own."""
    heads, heads_k, d, page, B = 8, 2, 128, 16, 3
    kp, vp, table = make_cache(B * 40, page, heads_k, d, 40, B)
    freqs = qg.rope_frequencies(d)
    pos, lengths = torch.zeros(B, dtype=torch.int64, device=DEV), torch.zeros(B, dtype=torch.int32, device=DEV)
    q, k, v = normal(B, heads, d, seed=1), normal(B, heads_k, d, seed=2), normal(B, heads_k, d, seed=3)

    def step():
        return qg.attention_paged(qg.cache_append(q, k, v, pos, kp, vp, table, freqs=freqs), kp, vp, table, lengths)
    step()
    torch.cuda.synchronize()
    graphs, outs = [], []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(step())
        graphs.append(g)
    for i, p in enumerate([0, 30, 511, 512, 600]):
        pos.copy_(torch.tensor([p, p // 2, p // 3], device=DEV))
        lengths.copy_((pos + 1).to(torch.int32))
        q.copy_(normal(B, heads, d, seed=10 + i))
        graphs[i % 2].replay()
        torch.cuda.synchronize()
        got = outs[i % 2].clone()
        want = step()
        torch.cuda.synchronize()
        assert torch.equal(got, want)


def test_refusals():
    kp, vp, table = make_cache(8, 16, 2, 64, 2, 3)
    q, k, v = normal(3, 4, 64), normal(3, 2, 64), normal(3, 2, 64)
    pos, freqs, n = torch.arange(3, device=DEV), qg.rope_frequencies(64), torch.ones(3, dtype=torch.int32, device=DEV)
    bad = [lambda: qg.rope_forward(q, k[:2], pos, freqs), lambda: qg.rope_forward(q, k, pos.int(), freqs), lambda: qg.rope_forward(q, k, pos, freqs.float()),
           lambda: qg.rope_forward(q, k, pos[:2], freqs), lambda: qg.rope_forward(q, k, pos, qg.rope_frequencies(66)), lambda: qg.rope_forward(q, k, pos, freqs, "both"),
           lambda: qg.rope_forward(q, k, pos, freqs, amplitude=float("nan")), lambda: qg.rope_forward(q, k, pos, freqs, out=(q[:1].expand(3, 4, 64), k)),
           lambda: qg.rope_frequencies(7), lambda: qg.rope_frequencies(8, base=-1.0), lambda: qg.rope_frequencies(8, factor=0.0),
           lambda: qg.rope_frequencies(8, context=100, low=4.0, high=4.0),
           lambda: qg.cache_append(q, k, v, pos, kp, vp[:4], table), lambda: qg.cache_append(q, k, v[:, :1], pos, kp, vp, table),
           lambda: qg.cache_append(q, k, v, pos, kp, vp, table.long()), lambda: qg.cache_append(q, k, v, pos, kp, vp, table, sequence=pos),
           lambda: qg.attention_paged(q[:2], kp, vp, table, n), lambda: qg.attention_paged(q[:, :3], kp, vp, table, n), lambda: qg.attention_paged(q, kp, vp, table, n.long()),
           lambda: qg.attention_paged(q, kp, vp, table, n, window=-1), lambda: qg.attention_paged(q, kp, vp, table, n, cap=float("inf")),
           lambda: qg.attention_paged(q, kp, vp, table, n, workspace=torch.empty(8, dtype=torch.uint8, device=DEV))]
    for call in bad:
        with pytest.raises(qg.QGError):
            call()
