"""metok_paged_evict on either side of the number of sequences up to which every CTA looks through the others' pages itself."""

import pytest
import torch

from paper_2506_02850_b200 import binding as B

from . import test_gpu_paged as P

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n_seqs", [31, 32, 33, 34, 64, 256, 257])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_sound_and_unsound_sequences(n_seqs, dtype):
    lens = [(37 * b) % 90 + (b % 7 > 0) for b in range(n_seqs)]
    lens[3], lens[5], lens[n_seqs - 1] = 60, 60, 75
    c = P.Cache(lens, 2, 64, 16, dtype, seed=n_seqs, layers=2)
    P.check_evict(c, 30, 4, 8)
    table, kv_len = c.block_table.clone(), c.kv_len.clone()
    table[3, 2] = table[n_seqs - 1, 4]                 # the last row of one's pages is another's
    table[5, 1] = table[5, 3]                          # one twice
    table[12, 0], kv_len[12] = c.n_pages, 20
    kv_len[20] = c.S_cap + 1
    out = {3, 5, 12, 20, n_seqs - 1}
    want = c.block_table.clone(), c.kv_len.clone()
    K, V, pos, mass = c.k.clone(), c.v.clone(), c.positions.clone(), c.mass.clone()
    got = B.metok_paged_evict(list(K.unbind(0)), list(V.unbind(0)), table, kv_len, mass, pos, 30, 4, 8)
    torch.cuda.synchronize()
    assert int(got["status"]) == -1
    K2, V2, pos2, mass2 = c.k.clone(), c.v.clone(), c.positions.clone(), c.mass.clone()
    good = B.metok_paged_evict(list(K2.unbind(0)), list(V2.unbind(0)), *want, mass2, pos2, 30, 4, 8)
    torch.cuda.synchronize()
    for b in range(n_seqs):
        if b in out:
            assert int(got["new_len"][b]) == int(kv_len[b]) and (got["keep_idx"][:, b] == -1).all()
            assert torch.equal(pos[:, b], c.positions[:, b]) and P.same(mass[:, b].contiguous(), c.mass[:, b].contiguous())
        else:
            assert int(got["new_len"][b]) == min(lens[b], 30) and torch.equal(got["keep_idx"][:, b], good["keep_idx"][:, b])
            assert torch.equal(pos[:, b], pos2[:, b]) and P.same(mass[:, b].contiguous(), mass2[:, b].contiguous())
        pages = [int(p) for p in c.table_np[b] if p < c.n_pages]
        ref = (c.k, c.v) if b in out else (K2, V2)
        assert P.same(K[:, pages].contiguous(), ref[0][:, pages].contiguous()) and P.same(V[:, pages].contiguous(), ref[1][:, pages].contiguous())
