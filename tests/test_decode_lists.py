"""Lists of pages that the attention is given: an empty axis, counts without
their lists, and lists that break their rules."""
import types

import pytest
import torch

from paper_2607_10582_amd import binding as B
from paper_2607_10582_amd.cache import MemDecay, PagedCache

D = 128


def test_an_empty_list_axis_is_not_every_page():
    # (an empty tensor's address is 0, which stands for "no list")
    md = MemDecay.__new__(MemDecay)
    md.cache, md._device, md.handle = types.SimpleNamespace(S=2, Hkv=2), -1, None
    blocks, count = torch.zeros((2, 2, 4), dtype=torch.int32), torch.zeros((2, 2), dtype=torch.int32)
    assert md._lists(blocks, count) == (blocks.data_ptr(), count.data_ptr(), 4)
    for empty in (blocks[:, :, :0], torch.zeros((2, 2, 0), dtype=torch.int32)):
        with pytest.raises(ValueError):
            md._lists(empty, count)


def _handle():
    c = PagedCache(L=1, Hq=4, Hkv=2, d=D, P=16, S=2, max_pages=4, n_phys=8, values=True, bounds=True)
    for pool in (c.k_pool, c.v_pool):
        pool.normal_()
    ones = torch.ones((2, 7))
    md = MemDecay(c, ones, ones, rho=0.9, alpha=1.0, tau_scale=2.0, pinned_mask=0)
    for s, n in enumerate((40, 7)):
        ids = list(range(4 * s, 4 * s + (n + 15) // 16))
        c.load_session(s, torch.randn((n, 1, 2, D)), [1] * n, ids, budget=n, clock=n)
        c.load_values(s, torch.randn((n, 1, 2, D)))
    return c, md


@pytest.mark.gpu
def test_attention_refuses_empty_and_half_given_lists():
    c, md = _handle()
    q, out = torch.randn((2, 4, D), device="cuda"), torch.full((2, 4, D), 3.0, device="cuda")
    nk = torch.randn((2, 2, D), device="cuda").to(torch.bfloat16)
    count = torch.zeros((2, 2), dtype=torch.int32, device="cuda")
    for kw in (dict(), dict(new_k=nk, new_v=nk)):
        with pytest.raises(ValueError):
            md.attend(0, q, out, blocks=torch.zeros((2, 2, 0), dtype=torch.int32, device="cuda"), block_count=count, **kw)
    with pytest.raises(ValueError):
        md.select_blocks(0, q, torch.zeros((2, 2, 0), dtype=torch.int32, device="cuda"), count, first=0, last=0)

    def raw(blocks, counts, most):   # past the Python checks
        return B.md_attend_token(md.handle, 0, B.ATTEND_ARGS.pack(q.data_ptr(), 4 * D, 0, 0, 0, c.v_pool.data_ptr(), blocks,
                                 counts, most, B.MD_F32, out.data_ptr(), 4 * D, 0, md._attend_ws.data_ptr()))

    blocks = torch.zeros((2, 2, 3), dtype=torch.int32, device="cuda")
    for a in ((0, count.data_ptr(), 0), (0, count.data_ptr(), 3), (blocks.data_ptr(), 0, 3), (blocks.data_ptr(), count.data_ptr(), 0)):
        with pytest.raises(B.MemDecayError) as e:
            raw(*a)
        assert e.value.status == B.MD_E_INVALID
    torch.cuda.synchronize()
    assert bool((out == 3.0).all())
    raw(0, 0, 0)
    raw(blocks.data_ptr(), count.data_ptr(), 3)                       # lists without entries: nothing is attended to
    torch.cuda.synchronize()
    assert not out.any() and md.device_status() == 0
