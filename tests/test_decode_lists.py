"""Lists of pages that the attention is given: an empty axis, counts without
their lists, and lists that break their rules."""
import types

import pytest
import torch

import decode_oracle as O
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


@pytest.mark.gpu
def test_what_counts_in_a_broken_list():
    # An entry counts where it names a page of the session and is above the
    # entry before it, whatever became of that one.  Equal keys, values that
    # tell the pages apart: the result is the mean over the tokens that count,
    # in whole numbers over their number (reciprocal and product, 2^-23); the
    # log-sum takes a logarithm of two units, a product and its constant (2^-22).
    c = PagedCache(L=1, Hq=4, Hkv=2, d=D, P=16, S=1, max_pages=8, n_phys=9, values=True)
    md = MemDecay(c, torch.ones((1, 7)), torch.ones((1, 7)), rho=0.9, alpha=1.0, tau_scale=2.0, pinned_mask=0)
    n = 7 * 16 - 5
    page = torch.arange(n) // 16
    values = (2.0 ** page)[:, None, None, None].expand(n, 1, 2, D)
    c.load_session(0, torch.zeros((n, 1, 2, D)), [1] * n, [3, 8, 1, 0, 7, 2, 5], budget=n, clock=n)
    c.load_values(0, values)
    for rows, counted in (([[5, 3, 4, 5], [0, 1 << 30, 1, 2]], [[5, 4, 5], [0, 2]]), ([[6, 6, 6, 6], [-1, 0, 7, 1]], [[6], [0]]),
                          ([[3, 2, 1, 0], [-5, -4, -3, 6]], [[3], [6]])):
        blocks = torch.tensor([rows], dtype=torch.int32, device="cuda")
        count = torch.full((1, 2), 4, dtype=torch.int32, device="cuda")
        out, lse = torch.zeros((1, 4, D), device="cuda"), torch.zeros((1, 4), device="cuda")
        md.attend(0, torch.ones((1, 4, D), device="cuda"), out, lse=lse, blocks=blocks, block_count=count)
        torch.cuda.synchronize()
        assert md.device_status() == B.MD_DEV_BAD_BLOCK
        for kv in range(2):
            v = torch.cat([values[page == o, 0, kv] for o in counted[kv]])
            ref, rl = O.attend(torch.ones((2, D)), torch.zeros_like(v), v)
            assert bool(((out[0, 2 * kv:2 * kv + 2].cpu() - ref).abs() <= 2.0 ** -23 * ref).all()), (rows, kv)
            assert bool(((lse[0, 2 * kv:2 * kv + 2].cpu() - rl).abs() <= 2.0 ** -22 * rl).all()), (rows, kv)
