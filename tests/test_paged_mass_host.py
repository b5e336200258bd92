"""The probability-mass check of the paged attention (tests/paged_mass.py) on the CPU: it takes what the roundings allow and
refuses planted mistakes."""

import numpy as np
import pytest
import torch

from paged_mass import KINDS, check_mass, classes, mass_batch, reference

CASES = [(9001, 4, 1, False), (9001, 4, 1, True), (40000, 2, 1, False), (5003, 3, 3, True)]


def batch(kind, keys, Hq, Hkv, fp8, new=1):
    return mass_batch(kind, [new], [keys], Hq, Hkv, 128, 128, 16, fp8, seed=keys, device="cpu")


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("keys,Hq,Hkv,fp8", CASES)
def test_mistakes_are_refused(kind, keys, Hq, Hkv, fp8):
    bt, scale = batch(kind, keys, Hq, Hkv, fp8), 128 ** -0.5
    o, _ = reference(bt, scale, True)
    check_mass(bt, torch.from_numpy(o).to(torch.bfloat16), scale, True)
    wrong = {"zero": np.zeros_like(o), "a tenth less": 0.9 * o, "two percent more": 1.02 * o, "half": 0.5 * o,
             "two classes exchanged": o[..., np.r_[1, 0, 2:128]], "first and last key": np.flip(o, axis=-1)}
    for a in (0, keys // 2, keys - 129):
        wrong[f"128 keys lost from {a}"] = reference(bt, scale, True, drop=(a, a + 128))[0]
    wrong["a half tile of 16 lost"] = reference(bt, scale, True, drop=(4096, 4112))[0]
    # A part of the keys with a weight that is five percent off.
    part = reference(bt, scale, True, drop=(keys // 3, keys))[0]
    share = (np.arange(128) <= classes(kind, keys, 128)[keys // 3]) if kind == "blocks" else np.arange(128) % 3 == 0
    wrong["a part's weight"] = np.where(share, 1.05 * o, o)
    assert not np.array_equal(part, o)
    for what, x in wrong.items():
        if kind == "residues" and what == "a half tile of 16 lost" and keys > 9001:
            continue  # 16 of 40 000 keys, one in each of 16 classes of 313: within the roundings of most
        with pytest.raises(AssertionError):
            check_mass(bt, x, scale, True, what)
            pytest.fail(f"{what} passes", pytrace=False)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("fp8", [False, True])
def test_the_roundings_are_taken(kind, fp8):
    """P rounded to 16 bits against a reference maximum, O rounded once."""
    bt, scale = batch(kind, 9001, 4, 1, fp8), 128 ** -0.5
    k = bt.values(bt.k_cache, bt.k_scale)
    rows = k[bt.table[0].numpy()[np.arange(9001) // 16], 0, np.arange(9001) % 16]
    x = (bt.q.double().numpy()[0] @ rows.T) * scale
    p = np.exp2((x - x[:, :128].max(axis=1, keepdims=True)) * 1.4426950408889634)
    rounded = torch.from_numpy(p * 128).to(torch.float16 if fp8 else torch.bfloat16).double().numpy() / 128
    hot = np.zeros((9001, 128))
    hot[np.arange(9001), classes(kind, 9001, 128)] = 1.0
    o = rounded @ hot / p.sum(axis=1, keepdims=True) * (bt.v_scale.double().item() if fp8 else 1.0)
    check_mass(bt, torch.from_numpy(o[None]).to(torch.bfloat16), scale, True)
