"""Infinite keys in a cache of e5m2, which keeps them: a score of -inf gives its key the weight 0 and nothing else, one of +inf and
one of 0 x inf make the row NaN, in a full block as in the open one, in each form of the attention over the cache."""
import pytest
import torch

from test_gpu_cache_attend_kernels import E5M2, FORMS, SHAPES, _attend, _case, _near, _reference

pytestmark = pytest.mark.gpu

# of the element that meets the infinity: 4 significant bits and 8, far below the row's largest and 0; either sign
PARTS = [1.0, -1.0, 1.1171875, -1.1171875, 0.0, 1.9921875, -1.9921875, 2.0 ** -20, -2.0 ** -20, 2.0 ** -8 * 1.4140625, -2.0 ** -8 * 1.4140625]


@pytest.mark.parametrize("value", [float("inf"), float("-inf")])
@pytest.mark.parametrize("b", [64, 128])
@pytest.mark.parametrize("shape", FORMS)
def test_infinite_keys(shape, b, value):
    n = SHAPES[shape][2]
    for back in (0, n // 2, n + 40, n + 270):  # in the open block; in full ones, that some rows see and that all do
        def change(q, K, V, pos):
            hq, n, _ = q.shape
            q[:, :, 3] = torch.tensor(PARTS, dtype=torch.bfloat16, device="cuda")[
                (torch.arange(n, device="cuda") + torch.arange(hq, device="cuda")[:, None]) % len(PARTS)]
            K[:, pos + n - 1 - back, 3] = value

        ses, c, keys, vals, q, pos = _case(shape, b, 21, E5M2, 8, change=change)
        assert keys[0, pos + n - 1 - back, 3] == value
        want, tol = _reference(q, keys, vals, pos)
        o = _attend(ses, c, q, pos)
        bad = torch.isnan(want)
        assert bad.any() and not bad.all()
        assert torch.equal(torch.isnan(o), bad), (back, int((torch.isnan(o) != bad).any(-1).sum()))
        _near(o, want, tol, where=~bad)


@pytest.mark.parametrize("shape", FORMS)
def test_infinities_of_several_keys(shape):
    # both infinities, two in one key, in tiles next to each other, beside an infinite value of V that some rows see; in place
    n = SHAPES[shape][2]

    def change(q, K, V, pos):
        q[:, ::2, 3] = -1.25
        q[:, 1::2, 3] = -1.2265625
        q[:, :, 70] = q[:, :, 70].abs() + 0.0078125
        K[:, 5, 3] = K[:, 64, 3] = K[:, pos, 3] = float("inf")
        K[:, 5, 70] = K[:, pos + n // 2, 70] = float("-inf")
        V[:, pos + n // 2, 9] = float("inf")

    ses, c, keys, vals, q, pos = _case(shape, 64, 13, E5M2, 9, change=change)
    at = pos + n // 2
    vals[:, at, 9] = 0
    want, tol = _reference(q, keys, vals, pos)
    assert not torch.isnan(want).any()
    ses.attend(c, q, pos, q)
    bad = torch.zeros(q.shape, dtype=torch.bool, device="cuda")
    bad[:, at - pos:, 9] = True  # weight 0 times an infinite value
    assert torch.equal(torch.isnan(q), bad)
    _near(q, want, tol, where=~bad)
