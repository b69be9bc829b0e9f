"""The statements that the operators around the expert layer are tested against, pinned on the CPU: the generator by its
published known answers, the derivatives and the balance gradient by differences."""
import numpy as np
import pytest
import torch

import block_ref as ref


@pytest.mark.parametrize("counter,key,want", [
    ((0, 0, 0, 0), (0, 0), (0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8)),
    ((0xFFFFFFFF,) * 4, (0xFFFFFFFF,) * 2, (0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD)),
    ((0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344), (0xA4093822, 0x299F31D0), (0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1)),
])
def test_generator_gives_its_published_answers(counter, key, want):
    assert tuple(int(v) for v in ref.philox4x32(counter, key)) == want


def test_mask_is_a_function_of_the_index():
    whole, factor = ref.keep_mask(5, 9, 0, 1000, 0.25)
    part, _ = ref.keep_mask(5, 9, 333, 100, 0.25)
    assert np.array_equal(whole[333:433], part) and factor == 65536 / 49152
    assert abs(ref.keep_mask(1, 2, 0, 1 << 18, 0.1)[0].mean() - 0.9) < 5 * (0.09 / (1 << 18)) ** 0.5
    assert not ref.keep_mask(1, 2, 0, 64, 1.0)[0].any() and ref.keep_mask(1, 2, 0, 64, 0.0)[0].all()


@pytest.mark.parametrize("a", range(5))
def test_slopes_by_differences(a):
    z = torch.linspace(-6, 6, 401, dtype=torch.float64) + 1e-3
    h = 1e-5
    diff = (ref.act(z + h, a) - ref.act(z - h, a)) / (2 * h)
    assert torch.allclose(diff, ref.act_slope(z, a), atol=1e-8)


def test_balance_gradient_by_differences():
    g = torch.Generator().manual_seed(3)
    a = torch.randn(12, 5, generator=g, dtype=torch.float64)
    topk = torch.topk(a, 2, 1).indices.int()
    live = torch.tensor([1, 1, 0, 1, 0, 0, 0, 0, 1, 0, 1, 1], dtype=torch.uint8)   # the second segment is empty
    loss, count, n, P, d = ref.balance(a, topk, 2, 0.3, 0.2, 3, live)
    assert n.tolist() == [3, 0, 3] and int(count.sum()) == 12 and torch.all(P[1] == 0)
    h = 1e-6
    for i in range(12):
        for j in range(5):
            up, down = a.clone(), a.clone()
            up[i, j] += h
            down[i, j] -= h
            diff = (ref.balance(up, topk, 2, 0.3, 0.2, 3, live)[0].sum() - ref.balance(down, topk, 2, 0.3, 0.2, 3, live)[0].sum()) / (2 * h)
            assert abs(float(diff - d[i, j])) < 1e-8
    uniform = ref.balance(torch.zeros(12, 5, dtype=torch.float64), topk, 2, 0.3, 0.0, 3, None)[0]
    assert abs(float(uniform[0]) - 0.3) < 1e-12
