"""The largest sizes that the operators of the uncompressed cache accept are launched whole."""
import pytest
import torch

from paper_2512_17917_amd import binding as kvr

pytestmark = [pytest.mark.gpu, pytest.mark.timeout(300)]
D = 128
BF = torch.bfloat16


def test_rotation_of_more_rows_than_a_launch_has_waves():
    """2^26 + 5 rows (17 GB of keys, in place): the last ones as a call on them alone gives them."""
    n = (1 << 26) + 5
    d = kvr.make_desc(1, 1, 1, 1, 1, BF)
    inv = (1e4 ** (-torch.arange(64, dtype=torch.float64) / 64)).cuda()
    turn = kvr.make_rotation(d, inv)
    k = torch.zeros(n, 1, D, dtype=BF, device="cuda")
    some = torch.randn(9, 1, D, generator=torch.Generator().manual_seed(1)).to(BF).cuda()
    k[:9], k[-9:] = some, some
    nc = torch.tensor([n], dtype=torch.int32).cuda()
    want = []
    for end in (9, n):
        alone = some.clone()
        kvr.kvr_rotate(d, turn, None, alone, None, 9, torch.tensor([0, 9], dtype=torch.int32).cuda(),
                       torch.tensor([end], dtype=torch.int32).cuda(), None, alone)
        want.append(alone)
    kvr.kvr_rotate(d, turn, None, k, None, n, torch.tensor([0, n], dtype=torch.int32).cuda(), nc, None, k)
    assert torch.equal(k[:9], want[0]) and torch.equal(k[-9:], want[1])
    assert not torch.equal(want[0], some)
