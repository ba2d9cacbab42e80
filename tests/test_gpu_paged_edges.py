"""Ends of the paged cache's documented ranges: contexts whose codes pass 2^32
words, layouts that run kernels of their own, infinities of small weight,
values at the pages' type's end."""
import numpy as np
import pytest

from tests import paged_ref as R
from tests.gpu_util import say

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from paper_2607_01065_amd import gsrq as B  # noqa: E402


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    B.load_library()


def _codeword_sums(codes, gain, shape, dtype):
    """Rows [tokens, G * d] of codes [tokens, M, G]: codewords rounded to float32, summed in float32 in stage order,
    rounded once: every bit as paged_restore documents it."""
    x = torch.zeros((codes.shape[0], shape.shape[1], shape.shape[3]), dtype=torch.float32, device=codes.device)
    g = torch.arange(shape.shape[1], device=codes.device)
    for m in range(shape.shape[0]):
        c = codes[:, m].long()
        x = x + gain[m][g, c][..., None] * shape[m][g, c]
    return x.flatten(1).to(dtype)


def test_restore_past_32_bit_code_words():
    """A context of 2^24 + 1000 tokens of 256 code words each, of which a few hundred have pages: the first tokens, where
    the words that are left just pass 2^32, and the last."""
    M, G, d, Hkv, hd, page = 64, 16, 8, 1, 128, 16
    L, words = 2 ** 24 + 1000, M * G // 4
    if torch.cuda.mem_get_info()[0] < 28 << 30:
        pytest.skip("less than 28 GiB free")
    g = torch.Generator(device="cuda").manual_seed(1)
    gain, shape = torch.rand((M, G, 256), generator=g, device="cuda"), torch.randn((M, G, 256, d), generator=g, device="cuda")
    codes = torch.zeros((1, L, words), dtype=torch.int32, device="cuda")
    per = -(-L // page)
    table = torch.full((1, per), -1, dtype=torch.int32)
    held = list(range(96)) + list(range(per - 8, per))               # tokens 0 .. 1535 and the last 120
    table[0, held] = torch.arange(len(held), dtype=torch.int32)
    at = torch.cat([torch.arange(page * i, page * i + page) for i in held])
    at = at[at < L].cuda()
    drawn = torch.randint(0, 256, (at.numel(), M, G), generator=g, device="cuda", dtype=torch.uint8)
    codes[0, at] = drawn.view(at.numel(), M * G).view(torch.int32)
    kp, vp = (torch.full((len(held), page, Hkv, hd), 9.0, dtype=torch.float16, device="cuda") for _ in range(2))
    say("restore", L, "tokens,", words, "words each")
    B.paged_restore(codes, codes, torch.tensor([L], dtype=torch.int32, device="cuda"), gain, shape, -gain, shape, kp, vp,
                    table.cuda())
    torch.cuda.synchronize()
    want = _codeword_sums(drawn, gain, shape, torch.float16)
    for pool, ref in ((kp, want), (vp, -want)):
        rows = pool.view(-1, hd)
        wrong = (rows[: at.numel()] != ref).any(1)
        assert not wrong.any(), f"{int(wrong.sum())} tokens, the first {int(at[wrong][0])}"
        assert torch.all(rows[at.numel():] == 9.0)                   # places behind the end


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("low", [8.0, 16.0])
@pytest.mark.parametrize("counts,lens,hd,until", [
    ([1], [100], 64, 33),                   # one piece; all of one wave's keys
    ([1, 3], [3000, 900], 128, 300),        # pieces that hold nothing else
    ([2], [2500], 256, 140),
    ([200], [500], 128, 140),               # many rows, tiles before all of them
    ([150, 1], [1500, 40], 64, 70),
    ([70], [1200], 256, 300),
])
def test_infinities_of_small_weight(counts, lens, hd, until, low, dtype):
    """Infinities and NaN in values that every row sees, at keys whose scores lie far below the others' (75 and 150 in
    log2 at heads of 64, twice that at 256): weights that are zero in float16, or in float32, are above zero all the
    same, so an infinity reaches the row, and where it is the first thing seen a later maximum does not undo it."""
    from tests.test_gpu_attn_paged import _case, _check
    c = _case(counts, lens, 4, 2, hd, 16, dtype)
    c["q"] = c["q"].abs()
    pages, page = c["kp"].shape[:2]
    bad = [float("inf"), -float("inf"), float("nan")]
    for b, L in enumerate(lens):
        n = counts[b]
        for t in range(min(until, L - n)):
            c["kp"][R.page_of(c["tab"], pages, page, b, t), t % page] = -low
        for i, t in enumerate((1, 2, min(until, L - n) - 1)):
            c["vp"][R.page_of(c["tab"], pages, page, b, t), t % page, :, 5 * i + b] = bad[i]
    got, lse = _check(c)
    assert torch.isinf(got).any() and torch.isnan(got).any() and torch.isfinite(lse).all()


def test_scores_of_nan_stay_with_their_row():
    """A row whose query or visible key is NaN gets NaN, whatever the values hold; its neighbours do not."""
    from tests.test_gpu_attn_paged import ORDER, _case
    for counts, lens in (([2], [700]), ([90], [300])):
        c = _case(counts, lens, 4, 2, 128, 16)
        ref = B.attn_paged(*(c[n].cuda() for n in ORDER))
        c["q"][1, 2, 7] = float("nan")
        got, lse = B.attn_paged(*(c[n].cuda() for n in ORDER), lse=True)
        assert torch.isnan(got[1, 2]).all() and torch.isnan(lse[1, 2])
        ref[1, 2] = got[1, 2] = 0
        assert torch.equal(got, ref)


@pytest.mark.parametrize("counts,lens,hd", [([1], [90], 64), ([3, 1], [2000, 700], 128), ([1], [9000], 256),
                                            ([200], [400], 128), ([40], [5000], 64), ([100], [700], 256)])
def test_values_at_the_types_end(counts, lens, hd):
    """All values are float16's largest.  Every 32nd key scores one more (in log2, less a little) than the others, whose
    weight lies just above the middle of two float16 numbers and is rounded up by 7/8 of half a step, 2^-11 of itself:
    the mean of these values must not become infinite by that."""
    from tests.test_gpu_attn_paged import _case, _check
    c = _case(counts, lens, 4, 2, hd, 16)
    pages, page = c["kp"].shape[:2]
    c["q"].zero_()
    c["kp"].zero_()
    c["q"][:, :, 0] = 1
    for b, L in enumerate(lens):
        for t in range(0, L, 32):
            c["kp"][R.page_of(c["tab"], pages, page, b, t), t % page, :, 0] = 1
    c["vp"].fill_(65504)
    c["vp"][..., 1::2] = -65504
    scale = (1 - np.log2(1 + 2.0 ** -11 * (1 + 2.0 ** -3))) * np.log(2.0)
    got, lse = _check(c, scale=float(np.float32(scale)))
    assert torch.isfinite(got).all()


@pytest.mark.parametrize("counts,lens,Hq,Hkv,hd,page,dtype,window", [
    ([1], [700], 40, 1, 128, 16, "f16", 0),                       # one token, more heads than a few-row workgroup's queries
    ([1, 1, 0, 1], [3000, 5, 9, 64], 64, 1, 64, 8, "bf16", 0),
    ([9, 1, 3], [500, 40, 3], 16, 4, 128, 16, "f16", 0),          # nine drafts of a group of four: 36 queries a key head
    ([1, 2], [900, 1200], 140, 1, 64, 32, "f16", 100),            # a token's heads in two workgroups
    ([1] * 70, [1 + 13 * b for b in range(70)], 66, 2, 64, 16, "bf16", 0),
])
def test_large_groups(counts, lens, Hq, Hkv, hd, page, dtype, window):
    """More than 32 queries per key head of very few tokens."""
    from tests.test_gpu_attn_paged import _case, _check
    _check(_case(counts, lens, Hq, Hkv, hd, page, dtype), window)


@pytest.mark.parametrize("lens,cap,Hkv,hd,d,K,M,page,held,rope", [
    ([900, 0, 30], 900, 2, 64, 8, 256, 2, 16, "f16", True),           # two stages resident in LDS
    ([600], 610, 3, 64, 16, 128, 2, 32, "bf16", True),                # the same, 7-bit codes across words
    ([600, 70], 600, 2, 128, 8, 8, 1, 16, "f16", True),               # one stage of 3-bit codes
    ([530], 530, 2, 256, 16, 32, 1, 8, "bf16", True),                 # of 5-bit codes, heads of 256
    ([77], 80, 5, 64, 8, 128, 1, 16, "f16", False),                   # of 7-bit codes, heads of 64
    ([641, 640, 5, 0], 641, 8, 128, 8, 256, 2, 16, "f16", True),      # chunks of 640 tokens, a code of its own each lane
    ([641, 100, 639, 64], 641, 8, 128, 16, 256, 4, 32, "bf16", True),  # the same, four lanes a code
    ([700, 1290], 1290, 8, 256, 64, 64, 6, 16, "bf16", True),         # 6-bit codes, heads of 256
])
def test_restore_layouts(lens, cap, Hkv, hd, d, K, M, page, held, rope):
    """Code layouts that run kernels of their own, within the tolerance derived in test_gpu_paged.test_restore."""
    from tests.test_gpu_paged import test_restore
    test_restore(lens, cap, Hkv, hd, d, K, M, page, held, rope)


@pytest.mark.parametrize("d,M", [(8, 1), (8, 2), (128, 12)])
def test_captured_restore_and_another_stream(d, M):
    """A restore captured and replayed on changed codes and lengths, among eager work, and on a stream of its own."""
    Hkv, hd, page, Bn, cap = 2, 128, 16, 2, 700
    G, per = Hkv * hd // d, -(-cap // page)
    g = torch.Generator(device="cuda").manual_seed(3)
    book = [torch.rand((M, G, 256), generator=g, device="cuda"), torch.randn((M, G, 256, d), generator=g, device="cuda")]
    codes = torch.randint(-2 ** 31, 2 ** 31 - 1, (Bn, cap, M * G * 8 // 32), generator=g, device="cuda", dtype=torch.int32)
    lens = torch.tensor([700, 333], dtype=torch.int32, device="cuda")
    tab = R.table(Bn, per, Bn * per).cuda()
    theta = (500000.0 ** (torch.arange(hd // 2, dtype=torch.float64) * (-2.0 / hd))).cuda()

    def pools():
        return [torch.zeros((Bn * per, page, Hkv, hd), dtype=torch.float16, device="cuda") for _ in range(2)]

    def restore(kp, vp, **kw):
        B.paged_restore(codes, codes, lens, *book, *book, kp, vp, tab, theta=theta, **kw)

    kept = pools()
    restore(*kept)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        restore(*kept)
    side = torch.cuda.Stream()
    for i in range(3):
        codes.copy_(torch.randint(-2 ** 31, 2 ** 31 - 1, codes.shape, generator=g, device="cuda", dtype=torch.int32))
        lens.sub_(torch.tensor([37, -41], dtype=torch.int32, device="cuda"))
        for pool in kept:
            pool.zero_()
        graph.replay()
        torch.cuda.synchronize()
        now, other = pools(), pools()
        restore(*now)
        side.wait_stream(torch.cuda.current_stream())
        restore(*other, stream=side)
        torch.cuda.synchronize()
        for a, b, c in zip(kept, now, other):
            assert torch.equal(a, b) and torch.equal(a, c) and a.any()


def test_restored_tokens_do_not_depend_on_the_chunks():
    """Chunks of 128 tokens in a short cache and of 640 in a long one give a token the same bits, rotation included."""
    Hkv, hd, page, d, M, n = 8, 128, 16, 128, 3, 700
    g = torch.Generator(device="cuda").manual_seed(5)
    book = [torch.rand((M, Hkv, 256), generator=g, device="cuda"), torch.randn((M, Hkv, 256, d), generator=g, device="cuda")]
    codes = torch.randint(-2 ** 31, 2 ** 31 - 1, (1, 9000, M * Hkv // 4), generator=g, device="cuda", dtype=torch.int32)
    theta = (500000.0 ** (torch.arange(hd // 2, dtype=torch.float64) * (-2.0 / hd))).cuda()
    lens = torch.tensor([n], dtype=torch.int32, device="cuda")
    tab = torch.arange(-(-n // page), dtype=torch.int32, device="cuda")[None]
    got = []
    for cap in (n, 1300, 9000):
        kp, vp = (torch.zeros((tab.numel(), page, Hkv, hd), dtype=torch.float16, device="cuda") for _ in range(2))
        c = codes[:, :cap].contiguous()
        B.paged_restore(c, c, lens, *book, *book, kp, vp, tab, theta=theta)
        got.append((kp, vp))
    for kp, vp in got[1:]:
        assert torch.equal(kp, got[0][0]) and torch.equal(vp, got[0][1]) and kp.any()


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("counts,lens,hd,window", [([1, 6], [77, 700], 128, 0), ([7], [133], 64, 40), ([4, 6], [500, 640], 256, 0),
                                                   ([90, 150], [90, 333], 128, 0), ([200], [300], 64, 70), ([70], [201], 256, 0)])
def test_what_a_row_does_not_see_changes_no_bit(counts, lens, hd, window, dtype):
    """Keys and values behind a sequence's end, in absent pages' places and, for the first rows of a call, in the tokens
    after theirs: large and small ones give the same bits, on keys that grow along the sequence, so that the maximum in
    use lags behind the largest score by up to 2^8."""
    from tests.test_gpu_attn_paged import ORDER, _case
    c = _case(counts, lens, 8, 2, hd, 16, dtype)
    pages, page = c["kp"].shape[:2]
    grow = torch.linspace(0.5, 2.0, max(lens)).to(c["kp"].dtype)
    used = torch.zeros((pages, page), dtype=torch.bool)
    late = []
    for b, L in enumerate(lens):
        for t in range(L):
            at = R.page_of(c["tab"], pages, page, b, t)
            used[at, t % page] = True
            c["kp"][at, t % page] *= grow[t]
        late += [(R.page_of(c["tab"], pages, page, b, t), t % page) for t in range(L - counts[b] // 2, L)]
    got = []
    for size in (0.0, 1.0, 30.0, -30.0):
        d = {n: c[n].clone() for n in ORDER}
        for name in ("kp", "vp"):
            d[name][~used] = size
            for at, i in late:
                d[name][at, i] = size
        got.append([x.cpu() for x in B.attn_paged(*(d[n].cuda() for n in ORDER), window=window, lse=True)])
    for b, n in enumerate(counts):
        first = slice(int(c["start"][b]), int(c["start"][b]) + n - n // 2)
        for other in got[1:]:
            assert torch.equal(other[0][first], got[0][0][first]) and torch.equal(other[1][first], got[0][1][first])
