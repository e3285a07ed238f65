"""Appending to the paged cache where the lists and the call do not count the same tokens."""
import numpy as np
import pytest
import torch

from oracle import paged_oracle as po
from paper_2512_12131_amd import binding as B
from test_gpu_kv_append import BF, DEV, lists, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("seqs,T", [([(5, 30)], 3), ([(1, 40), (60, 200)], 45), ([(900, 1000), (700, 700), (9, 20)], 1100)])
def test_the_first_tokens_of_a_batch(seqs, T):
    """A token's place is counted from its sequence's last one, whether or not the call has that."""
    Hkv, hd, page = 2, 128, 16
    c, every = make(seqs, Hkv, hd, page, seed=21)
    g = torch.Generator(device=DEV).manual_seed(2)
    q, k, v = (torch.randn((every, w * hd), generator=g, device=DEV).to(BF) for w in (4, Hkv, Hkv))
    cos, sin = B.lr_rope_table(1024, hd, device=DEV)
    cu, kv_len, table = lists(c)
    placed = np.array(po.places(cu, kv_len, table, page, c["k_cache"].shape[0], T))
    assert len(placed) == T
    t, pos, pg, row = (torch.from_numpy(placed[:, i].copy()).to(DEV) for i in (0, 2, 3, 4))
    want_k, want_v = c["k_cache"].clone(), c["v_cache"].clone()
    turn = lambda x, w: B.lr_rope_at(x[:T], cos, sin, w, hd, pos=pos.to(torch.int32))
    want_k[pg, row], want_v[pg, row] = turn(k, Hkv).view(T, Hkv, hd), v[:T].view(T, Hkv, hd)
    got = B.lr_kv_append(k[:T], v[:T], rope=(cos, sin), q=q[:T], H=4, **c)
    torch.cuda.synchronize()
    assert torch.equal(c["k_cache"], want_k) and torch.equal(c["v_cache"], want_v) and torch.equal(got, turn(q, 4))
