"""The block operators' oracle against what is known of them without it: published
words of the generator, differences, and inverses."""

import math

import pytest
import torch

from oracle import block


@pytest.mark.parametrize("counter,key,words", [
    # the published test vectors of Philox 4x32 in ten rounds
    ((0, 0, 0, 0), (0, 0), (0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8)),
    ((0xFFFFFFFF,) * 4, (0xFFFFFFFF,) * 2, (0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD)),
    ((0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344), (0xA4093822, 0x299F31D0), (0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1)),
])
def test_the_generators_words(counter, key, words):
    assert block.philox(counter, key) == words


def test_masks_do_not_depend_on_how_rows_are_cut():
    whole = block.kept(7, 16, 0.3, -5, 3)
    assert torch.equal(torch.cat([block.kept(3, 16, 0.3, -5, 3), block.kept(4, 16, 0.3, -5, 3, row0=3)]), whole)
    assert not torch.equal(block.kept(7, 16, 0.3, -5, 4), whole) and not torch.equal(block.kept(7, 16, 0.3, -4, 3), whole)
    share = float((block.kept(200, 64, 0.3, 1) == 0).double().mean())
    assert abs(share - 0.3) < 5 * math.sqrt(0.3 * 0.7 / 12800)
    assert (block.kept(3, 8, 1.0, 1) == 0).all() and (block.kept(3, 8, 0.0, 1) == 1).all()


def test_turning_back_is_the_inverse_and_the_gradient():
    g = torch.Generator().manual_seed(1)
    x, d = torch.randn((5, 3, 16), generator=g, dtype=torch.float64), torch.randn((5, 3, 16), generator=g, dtype=torch.float64)
    pos, freqs = torch.randint(0, 50, (5, 2), generator=g), torch.rand(7, generator=g)
    for nb in (False, True):
        y = block.turned(x, pos, freqs, (3, 4), 2, nb)[0]
        assert (block.turned(y, pos, freqs, (3, 4), 2, nb, back=True)[0] - x).abs().max() < 1e-13
        back = block.turned(d, pos, freqs, (3, 4), 2, nb, back=True)[0]
        assert abs(float((y * d).sum() - (x * back).sum())) < 1e-12


@pytest.mark.parametrize("rms", [False, True])
@pytest.mark.parametrize("parts", ["all", "pre", "y pre", "y post", "y gate"])
def test_the_norms_gradients_by_differences(parts, rms):
    g = torch.Generator().manual_seed(2)
    r = lambda *s: torch.randn(s, generator=g, dtype=torch.float64)  # noqa: E731
    v = {"x": r(3, 8)}
    if parts != "pre":
        v["y"] = r(3, 8)
    if parts in ("all", "y gate"):
        v["gate"] = r(8)
    if parts in ("all", "y post"):
        v["post_w"], v["post_b"] = r(8), r(8)
    if parts in ("all", "pre", "y pre"):
        v["pre_w"], v["pre_b"] = r(8), r(8)
    mask = block.kept(3, 8, 0.25, 9) if parts == "all" else None
    opt = {"rms": rms, "alpha": 0.7 if "y" in v else 1.0, "mask": mask}
    dh, dz = r(3, 8) if "y" in v else None, r(3, 8) if "pre_w" in v else None

    def value(v):
        o = block.add_norm(**v, **opt)
        return sum(float((o[k] * d).sum()) for k, d in (("h", dh), ("z", dz)) if d is not None)

    got = block.add_norm(**v, **opt, dh=dh, dz=dz)
    for name, t in v.items():
        for i in range(t.numel()):
            d = torch.zeros_like(t)
            d.view(-1)[i] = 1e-5
            want = (value(v | {name: t + d}) - value(v | {name: t - d})) / 2e-5
            assert abs(float(got["d" + name].reshape(-1)[i]) - want) < 1e-7 * (1 + abs(want)), (name, i)


def test_8_bit_floats_of_known_numbers():
    x = torch.zeros((1, 130))
    x[0, :7] = torch.tensor([448.0, -448.0, 17.0, 19.0, 2.0 ** -9, 2.0 ** -10, 3 * 2.0 ** -10])
    x[0, 128:] = torch.tensor([449.0, 0.0])
    q, e = block.fp8(x)
    assert e.tolist() == [[127, 128]]
    # ties to even: 17 between 16 and 18, 19 between 18 and 20, half of the least step, one and a half of it
    assert q[0, :7].tolist() == [448, -448, 16, 20, 2.0 ** -9, 0, 2 * 2.0 ** -9] and q[0, 128] == 224
    x[0, 3] = math.inf
    assert torch.isnan(block.unfp8(*block.fp8(x))[0, :128]).all() and block.unfp8(*block.fp8(x))[0, 128] == 448
