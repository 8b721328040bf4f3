"""Packed attention against float64: lengths from none to many, grouped heads, causal and not, caches, strides, rows of nobody."""
import math

import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
BF16, F32 = torch.bfloat16, torch.float32
NAN = float("nan")


@pytest.fixture(scope="module")
def dare():
    from paper_2605_08134_b200 import build
    build.build()
    from paper_2605_08134_b200 import dare as d
    return d


def make(lens, heads, kv_heads, hd, dtype, seed, gap=0, std=1.0, tail=3):
    """Packed q, k, v; `gap` rows of NaN behind every sequence's keys, `tail` query rows of nobody at the end."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    nq, nk = sum(a for a, _ in lens), sum(b + gap for _, b in lens)
    q = torch.full((nq + tail, heads, hd), NAN, device="cuda")
    q[:nq] = torch.randn((nq, heads, hd), generator=g, device="cuda") * std
    k, v = (torch.full((max(nk, 1), kv_heads, hd), NAN, device="cuda") for _ in range(2))
    q_begin, k_begin = [0], []
    at = 0
    for a, b in lens:
        q_begin.append(q_begin[-1] + a)
        k_begin.append(at)
        k[at:at + b] = torch.randn((b, kv_heads, hd), generator=g, device="cuda") * std
        v[at:at + b] = torch.randn((b, kv_heads, hd), generator=g, device="cuda") + 0.25
        at += b + gap
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    k_len = ints([b for _, b in lens]) if gap else None
    return q.to(dtype), k.to(dtype), v.to(dtype), ints(q_begin), ints(k_begin + ([] if gap else [at])), k_len


def check(lens, q, k, v, q_begin, k_begin, out, lse, causal, scale, untouched):
    """Every row of every sequence, and that the rows of nobody are as they were."""
    hd, group = q.shape[2], q.shape[1] // k.shape[1]
    bf16 = q.dtype == BF16
    qb, kb = q_begin.tolist(), k_begin.tolist()
    worst = 0.0
    for b, (nq, nk) in enumerate(lens):
        if nq == 0:
            continue
        rows = slice(qb[b], qb[b] + nq)
        qs = q[rows].double().transpose(0, 1)                                   # [heads, nq, hd]
        ks = k[kb[b]:kb[b] + nk].double().repeat_interleave(group, 1).transpose(0, 1)
        vs = v[kb[b]:kb[b] + nk].double().repeat_interleave(group, 1).transpose(0, 1)
        z = qs @ ks.transpose(1, 2) * scale
        mag = (qs.abs() @ ks.abs().transpose(1, 2) * scale).amax().item() if nk else 0.0
        if causal:
            z = z.masked_fill(torch.ones((nq, nk), dtype=torch.bool, device="cuda").triu(nk - nq + 1), -math.inf)
        want_lse = torch.logsumexp(z, -1) if nk else torch.full(z.shape[:2], -math.inf, dtype=torch.float64, device="cuda")
        w = torch.where(want_lse[..., None].isfinite(), (z - want_lse[..., None]).exp(), torch.zeros_like(z))
        want, size = w @ vs, w @ vs.abs()
        got, got_lse = out[rows].double().transpose(0, 1), lse[rows].double().transpose(0, 1)
        # a score: hd products summed in fp32 and scaled (the tensor core truncates: one ulp an addition), (2 hd + 8) 2^-24 of the sum of
        # magnitudes; 2^x to 2^-21 and its argument's rounding, 2^-23 of up to 3 mag; the sums over the keys, 2^-23 a key or
        # block of keys, at most (nk + 16) 2^-23
        eps = (2 * hd + 16) * 2.0 ** -24 * mag + 2.0 ** -20 + (nk + 16) * 2.0 ** -23
        # weights rounded to bf16 for the product: 2^-8 of each
        weights = 2.0 ** -8 if bf16 else 0.0
        bound = torch.finfo(q.dtype).eps / 2 * want.abs() * (1 + eps) + (weights + eps) * size
        assert bool(((got - want).abs() <= bound).all()), (b, ((got - want).abs() / bound.clamp(min=1e-30)).max().item())
        none = want_lse == -math.inf
        assert bool((got_lse[none] == -math.inf).all()) and bool((got[none] == 0).all())
        seen = ~none
        if bool(seen.any()):
            err = (got_lse[seen] - want_lse[seen]).abs()
            assert bool((err <= eps + 2.0 ** -22 * want_lse[seen].abs()).all()), (b, err.max().item())
    nobody = out[qb[-1]:]
    assert bool((nobody == untouched).all()) and bool((lse[qb[-1]:] == untouched).all())
    return worst


def run(dare, lens, heads, kv_heads, hd, dtype, causal, seed=0, gap=0, std=1.0, scale=None):
    q, k, v, qb, kb, kl = make(lens, heads, kv_heads, hd, dtype, seed, gap, std)
    out, status = torch.full_like(q, 7.0), torch.zeros(1, dtype=torch.int32, device="cuda")
    got, lse = dare.attention(q, k, v, qb, kb, k_len=kl, causal=causal, scale=scale, out=out, return_lse=True, status=status)
    assert got is out
    # (lse of the rows of nobody: allocated by the call, so a second one into a filled tensor through the C entry)
    lse2 = torch.full_like(lse, 7.0)
    cfg = dare.AttentionConfig(dare.C.sizeof(dare.AttentionConfig), dare.BF16 if dtype == BF16 else dare.F32, len(lens), heads, kv_heads,
                               hd, 1 if causal else 0, hd ** -0.5 if scale is None else scale, q.shape[0], k.shape[0],
                               *(s for t in (q, k, v, out) for s in t.stride()[:2]))
    work = torch.empty(dare.dare_attention_workspace_bytes(cfg), dtype=torch.uint8, device="cuda")
    again = torch.full_like(q, 7.0)
    st = dare.dare_attention(cfg, q.data_ptr(), k.data_ptr(), v.data_ptr(), qb.data_ptr(), kb.data_ptr(),
                             kl.data_ptr() if kl is not None else None, again.data_ptr(), lse2.data_ptr(), work.data_ptr(), work.numel(),
                             status.data_ptr(), torch.cuda.current_stream().cuda_stream)
    assert st == dare.OK
    n = sum(a for a, _ in lens)
    assert torch.equal(again, out) and torch.equal(lse2[:n], lse[:n])              # the same call gives the same bits
    check(lens, q, k, v, qb, kb, out, lse2, causal, hd ** -0.5 if scale is None else scale, 7.0)
    assert status.item() == dare.OK


LENGTHS = {
    "one": [(1, 1)],
    "tokens": [(1, 300), (1, 1), (1, 129), (1, 64), (1, 2000)],
    "none": [(0, 5), (3, 0), (64, 64), (0, 0), (1, 7), (5, 0)],
    "short": [(2, 2), (63, 63), (65, 65), (17, 40)],
    "uneven": [(130, 1000), (1, 3), (300, 300), (7, 511)],
    "few_keys": [(70, 10), (5, 5), (200, 33)],              # causal: the first queries see no key at all
}


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("heads,kv_heads,hd", [(1, 1, 128), (8, 2, 128), (14, 2, 64), (4, 4, 64), (7, 1, 128)])
@pytest.mark.parametrize("name", list(LENGTHS))
def test_bf16(dare, name, heads, kv_heads, hd, causal):
    run(dare, LENGTHS[name], heads, kv_heads, hd, BF16, causal, seed=len(name), gap=5)


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("heads,kv_heads,hd", [(8, 2, 64), (3, 3, 32), (14, 2, 128), (2, 1, 256)])
@pytest.mark.parametrize("name", list(LENGTHS))
def test_f32(dare, name, heads, kv_heads, hd, causal):
    run(dare, LENGTHS[name], heads, kv_heads, hd, F32, causal, seed=len(name), gap=5)


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("heads,kv_heads,hd", [(32, 8, 128), (16, 16, 64), (28, 4, 128)])
def test_prompts_fill_the_device(dare, heads, kv_heads, hd, causal):
    """Enough rows for 256 a CTA; packed without gaps, so that a block reaches into the next sequence."""
    run(dare, [(700, 700), (1, 1), (0, 0), (1531, 1531), (256, 256), (257, 900), (33, 20)], heads, kv_heads, hd, BF16, causal, seed=1)


def test_one_long_token(dare):
    run(dare, [(1, 40000)], 8, 1, 128, BF16, True, seed=2, gap=1)
    run(dare, [(1, 20011)], 4, 1, 64, F32, True, seed=2)


def test_many_sequences(dare):
    run(dare, [(i % 3, i % 7) for i in range(500)], 4, 2, 128, BF16, True, seed=3)
    run(dare, [(i % 3, i % 7) for i in range(150)], 2, 2, 32, F32, True, seed=3)


@pytest.mark.parametrize("causal", [False, True])
def test_few_keys_a_sequence(dare, causal):
    """On average; one sequence may hold nearly all of them."""
    run(dare, [(40, 490), (3, 0), (1, 1), (200, 12)], 6, 2, 64, F32, causal, seed=5)
    run(dare, [(128, 128)], 4, 4, 256, F32, causal, seed=6)
    run(dare, [(300, 100), (5, 156)], 8, 1, 32, F32, causal, seed=7)


def test_many_prompts(dare):
    """More sequences than the form with 256 rows a CTA is meant for."""
    run(dare, [(129 + i % 5, 129 + i % 7) for i in range(300)], 4, 2, 128, BF16, True, seed=8)


def test_large_scores(dare):
    """Scores of some hundreds: the weights of all but a few keys vanish, the maximum moves often."""
    run(dare, [(200, 900), (1, 700)], 8, 2, 128, BF16, False, seed=4, std=4.0)
    run(dare, [(200, 900), (1, 700)], 8, 2, 128, BF16, True, seed=4, std=1.0, scale=2.0)
    run(dare, [(64, 400)], 2, 2, 64, F32, True, seed=4, std=4.0)


def test_bf16_on_the_cuda_cores(dare):
    """Heads that the tensor cores do not take, and rows off the 16-byte grid."""
    run(dare, [(5, 77), (40, 40)], 4, 2, 32, BF16, True, seed=5)
    run(dare, [(5, 77), (40, 40)], 4, 2, 256, BF16, False, seed=5)
    lens = [(9, 50), (30, 30)]
    q, k, v, qb, kb, _ = make(lens, 4, 2, 128, BF16, 6)
    odd = [torch.zeros(t.numel() + 1, dtype=BF16, device="cuda")[1:].view(t.shape).copy_(t) for t in (q, k, v)]
    out, lse = dare.attention(*odd, qb, kb, causal=True, out=torch.full_like(q, 7.0), return_lse=True)
    lse[39:] = 7.0
    check(lens, q, k, v, qb, kb, out, lse, True, 128 ** -0.5, 7.0)


@pytest.mark.parametrize("hd", [64, 128])
def test_strides(dare, hd):
    """Views of a fused projection, head-major caches, head-major output, one key/value head shared by stride."""
    lens = [(100, 100), (1, 1), (37, 37)]
    q, k, v, qb, kb, _ = make(lens, 8, 2, hd, BF16, 7, tail=0)
    fused = torch.cat((q, k, v), 1)
    fq, fk, fv = fused[:, :8], fused[:, 8:10], fused[:, 10:]
    want, want_lse = dare.attention(q, k, v, qb, kb, causal=True, return_lse=True)
    check(lens, q, k, v, qb, kb, want, want_lse, True, hd ** -0.5, 0.0)
    got, lse = dare.attention(fq, fk, fv, qb, kb, causal=True, return_lse=True)
    assert torch.equal(got, want) and torch.equal(lse, want_lse)
    hm = lambda t: t.transpose(0, 1).contiguous().transpose(0, 1)
    out = torch.empty((8, q.shape[0], hd), dtype=BF16, device="cuda").transpose(0, 1)
    dare.attention(hm(q), hm(k), hm(v), qb, kb, causal=True, out=out)
    assert torch.equal(out, want)
    dare.attention(q, hm(k), v, qb, kb, causal=True, out=out)
    assert torch.equal(out, want)
    # keys that overlap: every row of a sliding window over one line
    line = torch.randn(138 * 8 + 2 * hd, device="cuda").to(BF16)
    slide = line.as_strided((138, 2, hd), (8, hd, 1))
    got, lse = dare.attention(q, slide, slide, qb, kb, causal=True, return_lse=True)
    check(lens, q, slide, slide, qb, kb, got, lse, True, hd ** -0.5, 0.0)
    one_k, one_v = k[:, :1], v[:, :1]
    shared = dare.attention(q, one_k.expand(-1, 2, -1), one_v.expand(-1, 2, -1), qb, kb, causal=True)       # head stride 0
    assert (shared.float() - dare.attention(q, one_k, one_v, qb, kb, causal=True).float()).abs().max().item() <= 2.0 ** -5


def test_infinities_and_nan_outside_the_mask(dare):
    """What lies behind a sequence's keys, in a neighbour's or in tiles that causality hides whole, never comes through."""
    for dtype, hd in ((BF16, 128), (BF16, 64), (F32, 64)):
        lens = [(40, 40), (1, 100), (20, 20)]
        q, k, v, qb, kb, _ = make(lens, 4, 2, hd, dtype, 8)
        want, lse = dare.attention(q, k, v, qb, kb, causal=True, return_lse=True)
        want, lse = want.clone(), lse.clone()
        k[40:140], v[40:140] = float("inf"), NAN                                # the second sequence is broken
        got, lse2 = dare.attention(q, k, v, qb, kb, causal=True, return_lse=True)
        ok = list(range(40)) + list(range(41, 61))
        assert torch.equal(got[ok], want[ok]) and torch.equal(lse2[ok], lse[ok])
        assert bool(got[40].isnan().all())
        k[39, :, 0] = float("inf")                                              # the last key of the first: hidden from all queries but one
        got, _ = dare.attention(q, k, v, qb, kb, causal=True, return_lse=True)
        assert torch.equal(got[:39], want[:39])


def test_offsets_past_32_bits(dare):
    """A cache of 2.3 million rows of 8 x 128: elements past 2^31."""
    rows, kvh, hd = 2_300_000, 8, 128
    g = torch.Generator(device="cuda").manual_seed(9)
    k, v = (torch.empty((rows, kvh, hd), dtype=BF16, device="cuda") for _ in range(2))
    begin, lens = [0, 2_200_000, rows - 333], [(1, 200), (3, 500), (130, 333)]
    for at, (_, n) in zip(begin, lens):
        k[at:at + n] = torch.randn((n, kvh, hd), generator=g, device="cuda").to(BF16)
        v[at:at + n] = torch.randn((n, kvh, hd), generator=g, device="cuda").to(BF16)
    q = torch.randn((134, 16, hd), generator=g, device="cuda").to(BF16)
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    qb, kb, kl = ints([0, 1, 4, 134]), ints(begin), ints([n for _, n in lens])
    out, lse = dare.attention(q, k, v, qb, kb, k_len=kl, causal=True, return_lse=True)
    check(lens, q, k, v, qb, kb, out, lse, True, hd ** -0.5, 0.0)
    big = torch.empty((2 * (1 << 30) // (8 * 128) + 200, 8, 128), dtype=BF16, device="cuda")      # and queries and outputs
    big[-134:] = q[:, :8]
    qb2 = ints([big.shape[0] - 134 + x for x in (0, 1, 4, 134)])
    out2, lse2 = dare.attention(big, k, v, qb2, kb, k_len=kl, causal=True, out=torch.zeros_like(big), return_lse=True)
    check(lens, big, k, v, qb2, kb, out2, lse2, True, hd ** -0.5, 0.0)
    assert not bool(out2[:-134].any())


@pytest.mark.parametrize("dtype,hd", [(BF16, 128), (F32, 64)])
def test_slices_outside_the_arrays(dare, dtype, hd):
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    q, k, v, qb, kb, _ = make([(4, 30), (4, 30), (4, 30)], 4, 2, hd, dtype, 10, tail=0)
    want = dare.attention(q, k, v, qb, kb)
    for bad_qb, bad_kb, bad_kl, skipped in ((qb, ints([0, 30, 60, 91]), None, (8, 12)), (qb, ints([0, -1, 60]), ints([30, 30, 30]), (4, 8)),
                                            (qb, ints([0, 30, 60]), ints([30, -2, 30]), (4, 8)), (ints([0, 4, 8, 13]), kb, None, (8, 12)),
                                            (qb, ints([0, 30, 60]), ints([30, 30, 2 ** 31 - 1]), (8, 12))):
        status, out = torch.zeros(1, dtype=torch.int32, device="cuda"), torch.full_like(q, 7.0)
        dare.attention(q, k, v, bad_qb, bad_kb, k_len=bad_kl, out=out, status=status)
        assert status.item() == dare.ERR_DEVICE_CHECK
        assert bool((out[skipped[0]:skipped[1]] == 7.0).all())
        keep = [i for i in range(12) if not skipped[0] <= i < skipped[1]]
        assert torch.allclose(out[keep].float(), want[keep].float(), atol=2.0 ** -6)      # (shares cut elsewhere: other roundings)


@pytest.mark.parametrize("dtype,hd,n", [(BF16, 128, 30), (F32, 64, 30), (F32, 64, 1500), (BF16, 64, 1500)])
def test_slices_that_run_backwards(dare, dtype, hd, n):
    """Offsets that go back and forth: the slices that run backwards are skipped, and those that then overlap are each right."""
    q, k, v, qb, kb, _ = make([(70, n)], 4, 2, hd, dtype, 12, tail=2)
    want = dare.attention(q, k, v, qb, kb)[:70]
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    status, out = torch.zeros(1, dtype=torch.int32, device="cuda"), torch.full_like(q, 7.0)
    dare.attention(q, k, v, ints([0, 70] * 40), ints([0] * 79), k_len=ints([n] * 79), out=out, status=status)
    assert status.item() == dare.ERR_DEVICE_CHECK
    bad = (out[:70].float() - want.float()).abs() > 2.0 ** -6
    rows = bad.flatten(1).any(1)
    assert not bool((rows & (out[:70] != 7.0).flatten(1).all(1)).any())          # (a row may be left out)
    assert bool((out[70:] == 7.0).all())


def test_streams_and_graphs(dare):
    lens = [(1, 3000), (1, 77), (1, 1500), (1, 1)]
    q, k, v, qb, kb, _ = make(lens, 32, 8, 128, BF16, 11, tail=0)
    want = dare.attention(q, k, v, qb, kb, causal=True)
    # two calls at once on two streams, each with its own workspace
    streams, outs = [torch.cuda.Stream() for _ in range(2)], []
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    for _ in range(5):
        for s in streams:
            with torch.cuda.stream(s):
                outs.append(dare.attention(q, k, v, qb, kb, causal=True))
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for o in outs)
    # captured, replayed with other lengths on the device
    kl = torch.tensor([b for _, b in lens], dtype=torch.int32, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = dare.attention(q, k, v, qb, kb[:4], k_len=kl, causal=True)
    graph.replay()
    assert torch.equal(out, want)
    kl.copy_(torch.tensor([5, 60, 1000, 0], dtype=torch.int32))
    graph.replay()
    assert torch.equal(out, dare.attention(q, k, v, qb, kb[:4], k_len=kl, causal=True))
    assert bool((out[3] == 0).all())


def test_nothing_to_do(dare):
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    empty = torch.empty((0, 4, 128), dtype=BF16, device="cuda")
    k = torch.randn((8, 2, 128), device="cuda").to(BF16)
    assert dare.attention(empty, k, k, ints([0, 0]), ints([0, 8])).shape == (0, 4, 128)
    q = torch.randn((3, 4, 128), device="cuda").to(BF16)
    none = torch.empty((0, 2, 128), dtype=BF16, device="cuda")
    out, lse = dare.attention(q, none, none, ints([0, 3]), ints([0, 0]), return_lse=True)
    assert not bool(out.any()) and bool((lse == -math.inf).all())
