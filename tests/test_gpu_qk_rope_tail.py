"""Elements from rotary_dim on are normed and no more, whatever lies beside them: no tolerance without a norm, bit for bit."""
import pytest
import torch

from paper_2601_19278_b200 import binding as b
from test_gpu_kv8 import DEV
from test_gpu_qk_rope import EPS, THETA, TYPES, check

pytestmark = pytest.mark.gpu


def rotated(q, k, rotary, interleaved, gain, lens):
    qo, ko = torch.full_like(q, 7.0), torch.full_like(k, 7.0)
    b.qk_norm_rope(q, k, qo, ko, b.rope_frequencies(THETA, rotary, DEV), seq_lens=torch.tensor(lens, dtype=torch.int32, device=DEV), q_norm=gain,
                   k_norm=gain, eps=EPS, interleaved=interleaved)
    torch.cuda.synchronize()
    return qo, ko


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("d,rotary", [(128, 64), (128, 16), (128, 112), (64, 32), (64, 48)])
def test_the_tail_of_a_head_stays_bit_for_bit(dtype, interleaved, d, rotary):
    """Infinities, NaN, zeros of both signs and the largest values among it; the rotated part does not notice them either."""
    g = torch.Generator().manual_seed(d + rotary)
    lens = [1000, 5]
    q, k = (torch.randn(2, 3, n, d, generator=g) * 3 for n in (5, 2))
    for x in (q, k):
        x[..., rotary::3] = -0.0
        x[0, 0, 0, rotary], x[0, 1, 1, d - 1], x[1, 2, 0, rotary + 9] = float("inf"), float("-inf"), float("nan")
        x[1, 0, 1, rotary + 8] = torch.finfo(TYPES[dtype]).max
    q, k = (x.to(TYPES[dtype]).to(DEV) for x in (q, k))
    bits = torch.int32 if dtype == "fp32" else torch.int16
    for got, x in zip(rotated(q, k, rotary, interleaved, None, lens), (q, k)):
        tail, want = got[..., rotary:], x[..., rotary:]
        assert torch.equal(tail.isnan(), want.isnan())                       # (which NaN it is says nothing)
        assert torch.equal(tail.nan_to_num(0.0, float("inf"), float("-inf")).view(bits), want.nan_to_num(0.0, float("inf"), float("-inf")).view(bits))
        clean = x.clone()
        clean[..., rotary:] = 0.0
        got = got.clone()
        got[..., rotary:] = 0.0
        check(got, clean, None, [[n + r for r in range(3)] for n in lens], rotary, interleaved, dtype)


@pytest.mark.parametrize("interleaved", [False, True])
def test_a_norm_over_an_infinity_in_the_tail_leaves_nan_there_alone(interleaved):
    """mean(x^2) is infinite, its root's inverse 0: 0 times infinity is NaN, every other element 0."""
    q = torch.ones(1, 1, 2, 128, dtype=torch.bfloat16, device=DEV)
    q[0, 0, 0, 100] = float("inf")
    got, _ = rotated(q, q.clone(), 64, interleaved, torch.ones(128, dtype=torch.bfloat16, device=DEV), [9])
    want = torch.zeros(128, dtype=torch.bool, device=DEV)
    want[100] = True
    assert torch.equal(got[0, 0, 0].isnan(), want) and bool((got[0, 0, 0][~want] == 0).all()) and bool(got[0, 0, 1].isfinite().all())
