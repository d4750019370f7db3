"""metok_paged_append with offsets that descend, or leave the new rows: which sequences are extended, and by what."""

import pytest
import torch

from paper_2506_02850_b200 import binding as B

from . import test_gpu_paged as P

pytestmark = pytest.mark.gpu


def append(lens, offsets, n_new, dtype, untouched=False):
    c = P.Cache(lens, 2, 64, 16, dtype, seed=2, room=n_new)
    kn, vn = (torch.randn((2, n_new, 64), generator=c.g, device="cuda").to(dtype) for _ in range(2))
    k, v, pos, mass = c.k[0].clone(), c.v[0].clone(), c.positions[0].clone(), c.mass[0].clone()
    got = B.metok_paged_append(kn, vn, k, v, c.block_table, c.kv_len, torch.tensor(offsets, dtype=torch.int32, device="cuda"), pos, None, mass)
    torch.cuda.synchronize()
    new_len = got["new_len"].tolist()
    if untouched:
        assert P.same(k, c.k[0]) and P.same(v, c.v[0]) and torch.equal(pos, c.positions[0]) and P.same(mass, c.mass[0])
    # rows that were there, and every row that a sequence is said to have got
    for b, n in enumerate(lens):
        for r in range(new_len[b]):
            page = int(c.table_np[b, r // c.page])
            i = offsets[b] + r - n
            want = (c.k[0][page, :, r % 16], c.v[0][page, :, r % 16]) if r < n else (kn[:, i], vn[:, i])
            assert P.same(k[page, :, r % 16].contiguous(), want[0].contiguous()) and P.same(v[page, :, r % 16].contiguous(), want[1].contiguous()), (b, r)
        assert torch.equal(mass[b, :n], c.mass[0, b, :n]) and torch.equal(pos[b, :n], c.positions[0, b, :n])
        assert (mass[b, n:new_len[b]] == 0).all()
        at = int(c.positions[0, b, n - 1]) + 1 if n else 0
        assert pos[b, n:new_len[b]].tolist() == list(range(at, at + new_len[b] - n))
    return int(got["status"]), new_len


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("lens,offsets,n_new", [([5, 6, 7], [0, 9, 4, 8], 8), ([20, 30, 40, 10, 50], [0, 4, 2, 12, 16, 20], 20), ([20, 0, 1], [0, 5, 3, 8], 8),
                                                ([3, 3, 3, 3], [4, 0, 4, 8, 12], 12), ([3] * 70, list(range(60)) + [50] + list(range(61, 71)), 70),
                                                ([2, 2], [0, 2 ** 31 - 1, -2 ** 31], 6), ([2, 2, 2], [0, 3, 6, 5], 6)])
def test_offsets_that_descend_extend_nothing(dtype, lens, offsets, n_new):
    assert append(lens, offsets, n_new, dtype, untouched=True) == (-1, lens)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("lens,offsets,n_new,new_len", [([20, 30, 40], [0, 4, 8, 13], 12, [24, 34, 40]), ([20, 30, 40], [-1, 4, 8, 12], 12, [20, 34, 44]),
                                                        ([20, 30, 40], [0, 4, 13, 13], 12, [24, 30, 40]), ([20, 30, 40], [2, 2, 8, 11], 12, [20, 36, 43])])
def test_of_ascending_offsets_only_what_leaves_is_left_out(dtype, lens, offsets, n_new, new_len):
    status, got = append(lens, offsets, n_new, dtype)
    assert got == new_len and status == (0 if offsets[0] >= 0 and offsets[-1] <= n_new else -1)
