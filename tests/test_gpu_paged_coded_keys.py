"""Keys of a paged session that are also kept as codes: coded after the norm of
their heads and before the rotation, as paged_restore takes them; and the
README's example, as it stands there, with rows in the pages' type."""
import os
import re

import pytest

from tests import paged_ref as R

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from paper_2607_01065_amd import gsrq as B  # noqa: E402


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    B.load_library()


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_normed_keys_come_back_from_codes(dtype):
    """The pages that a restore fills differ from those that the append filled by the codes' error alone, which a rotation
    does not change in size, and by roundings: two to the pages' type, and 2^-19 for either rotation."""
    Hkv, hd, page, d, M = 2, 64, 16, 8, 4
    T, G, dt = 77, Hkv * hd // d, R.TYPES[dtype]
    g = torch.Generator().manual_seed(6)
    k, v = (torch.randn((T, Hkv, hd), generator=g).to(dt).cuda() for _ in range(2))
    w = (1 + 0.3 * torch.randn(hd, generator=g)).cuda()
    theta = (500000.0 ** (torch.arange(hd // 2, dtype=torch.float64) * (-2.0 / hd))).cuda()
    gain = (2.0 * 0.4 ** torch.arange(M)[:, None, None] * torch.rand((M, G, 256), generator=g)).cuda()
    shape = torch.randn((M, G, 256, d), generator=g)
    shape = (shape / shape.norm(dim=-1, keepdim=True)).cuda()
    per = -(-T // page)
    tab, lens = R.table(1, per, per + 1).cuda(), torch.tensor([T], dtype=torch.int32, device="cuda")
    pools = [torch.zeros((per + 1, page, Hkv, hd), dtype=dt, device="cuda") for _ in range(4)]
    B.paged_append(k, v, *pools[:2], tab, torch.tensor([0, T], dtype=torch.int32, device="cuda"), lens, theta=theta, k_norm=w)
    x = k.float()
    normed = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6) * w
    codes, lost = [], []
    for rows in (normed, v.float()):
        c, e = B.encode(rows.reshape(T, -1), gain, shape, residual=True)
        codes.append(c.view(1, T, -1))
        lost.append(e.view(T, Hkv, hd).double().norm(dim=-1))
    B.paged_restore(*codes, lens, gain, shape, gain, shape, *pools[2:], tab, theta=theta)
    at = tab[0].long()
    rel, sub = R.half_step(dt)
    for i in range(2):
        a, b = (pools[j][at].view(-1, Hkv, hd)[:T].double() for j in (i, i + 2))
        room = lost[i] + (rel + 2.0 ** -18) * (a.norm(dim=-1) + b.norm(dim=-1)) * 1.01 + 16 * sub
        assert torch.all((a - b).norm(dim=-1) <= room)


def test_readme_example():
    """The block of the README that serves over pages, for a model whose keys are in the pages' type."""
    text = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "README.md")).read()
    block = next(b for b in re.findall(r"```python\n(.*?)```", text, re.S) if "paged_append" in b)
    block = re.sub(r"^(table|q_start, seq_len) = \.\.\..*$", "", block, flags=re.M)
    Hkv, pages, T = 2, 9, 40
    D = Hkv * 128
    g = torch.Generator(device="cuda").manual_seed(7)
    k, v, q = (torch.randn((T, h, 128), generator=g, device="cuda").bfloat16() for h in (Hkv, Hkv, 4))
    gain, shape = torch.rand((1, D // 8, 256), generator=g, device="cuda"), torch.randn((1, D // 8, 256, 8), generator=g, device="cuda")
    codes = torch.randint(-2 ** 31, 2 ** 31 - 1, (2, 64, D // 32), generator=g, device="cuda", dtype=torch.int32)
    names = dict(torch=torch, B=B, k=k, v=v, q=q, T=T, Hkv=Hkv, pages=pages, gain=gain, shape=shape, k_codes=codes, v_codes=codes,
                 k_gain=gain, v_gain=gain, k_shape=shape, v_shape=shape, table=torch.arange(8, dtype=torch.int32, device="cuda").view(2, 4),
                 q_start=torch.tensor([0, 30, T], dtype=torch.int32, device="cuda"),
                 seq_len=torch.tensor([30, 64], dtype=torch.int32, device="cuda"),
                 v_pages=torch.zeros((pages, 16, Hkv, 128), dtype=torch.bfloat16, device="cuda"))
    exec(block, names)
    torch.cuda.synchronize()
    assert names["out"].shape == (T, 4, 128) and names["out"].dtype == torch.bfloat16
    assert names["codes"].shape == (T, D // 32)
