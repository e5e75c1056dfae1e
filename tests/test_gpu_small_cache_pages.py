"""Page entries outside the pool in the calls that write the weights of cached tokens: nothing but the tokens of good pages is written."""
import numpy as np
import pytest
import torch

from test_gpu_small_cache import attention_case, host, i32

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2511_03983_b200 import binding
    binding.lib()
    return binding


@pytest.mark.parametrize("q8", [True, False])
@pytest.mark.parametrize("D,page,lens,H,NH,NKV", [(16, 16, [100, 70], 4, 8, 2), (64, 32, [300, 33], 4, 8, 2), (64, 16, [130, 47], 12, 12, 1),
                                                  (128, 16, [90, 1000], 3, 8, 2)])
def test_weights_of_tokens_whose_page_is_bad_are_written_nowhere(B, D, page, lens, H, NH, NKV, q8):
    """The pool's first page is a sequence's own (not the one with bad entries): its weights and positions are those of a call
    without bad entries, and so are all others that have a page; twelve heads on a position take two passes."""
    gen = torch.Generator().manual_seed(D + page)
    c = attention_case(gen, D, page, 1, lens, H, NH, NKV, q8)
    good = [list(r) for r in c["table"]]
    zero = next((i, j) for i, r in enumerate(good) for j, p in enumerate(r) if p == 0) if any(0 in r for r in good) else None
    if zero is None:                                  # the spare pages took it: the first sequence's first page becomes page 0
        old, zero = good[0][0], (0, 0)
        good[0][0] = 0
        c["k"][0] = c["k"][old]
        if q8:
            c["scales"][0] = c["scales"][old]
    lse = torch.zeros(1, H, 2, device="cuda")
    prior = torch.rand(c["pool"], c["KV"], page, generator=gen).cuda()
    new = [lens[0] // 2, lens[1]]                     # many new tokens: their positions are written

    def call(table, in_place):
        w = prior.clone() if in_place else torch.full_like(prior, -3.0)
        pos = torch.full(prior.shape, -9, dtype=torch.int32, device="cuda")
        B.twist_attn_weights(B.attn_weights_args(
            B.BF16, 1, 2, H, c["KV"], D, NH, NKV, q=c["q"].cuda(), lse=lse, k_cache=c["k"], scales=c["scales"], page_table=i32([table]),
            kv_len=i32([lens]), new_len=i32([new]), head_idx=i32(c["idx"]), kv_pos=i32(c["kv_pos"]), prior=w if in_place else prior,
            weights=w, slot_pos=pos))
        return host(w), pos.cpu().numpy(), B.twist_device_status()

    for in_place in (False, True):
        want, where, status = call(good, in_place)
        assert status == 0
        for entry in (-1, c["pool"], 10 ** 6, -2 ** 31):
            b = 1 - zero[0]                           # the other sequence gets the bad entries
            used = -(-lens[b] // page)
            for bad in ([0], [used - 1], list(range(used)), list(range(1, used, 2))):
                table = [list(r) for r in good]
                lost = [p for j, p in enumerate(table[b]) if j in bad]
                table[b] = [entry if j in bad else p for j, p in enumerate(table[b])]
                got, at, status = call(table, in_place)
                assert status == (B.ERR_BAD_INDEX if lost else 0)
                rest = np.setdiff1d(np.arange(c["pool"]), lost)
                assert np.array_equal(got[rest], want[rest]) and np.array_equal(at[rest], where[rest]), (entry, bad, in_place)
                assert np.all(got[lost] == (host(prior)[lost] if in_place else -3.0)) and np.all(at[lost] == -9)


@pytest.mark.parametrize("D,N", [(8, 70), (16, 40), (32, 300), (64, 129), (128, 200)])
def test_positions_without_heads_are_left_as_they_were(B, D, N):
    """Both heads read position 1 of three: the others' weights and positions stay, of prompts and of a step."""
    gen = torch.Generator().manual_seed(D)
    page, KV, H = 16, 3, 2
    pages = -(-N // page)
    table = i32([[list(range(1, pages + 1))]])
    heads = dict(head_idx=i32([[2, 3]]), kv_pos=i32([[0, 1, 2]]))
    x = torch.randn(1, N, (H + 2 * KV) * D, generator=gen).to(torch.bfloat16).cuda()
    k = torch.randn(pages + 2, KV, page, D, generator=gen).to(torch.bfloat16).cuda()

    def check(call):
        w = torch.full((pages + 2, KV, page), -3.0, device="cuda")
        pos = torch.full(w.shape, -9, dtype=torch.int32, device="cuda")
        call(w, pos)
        assert B.twist_device_status() == 0
        mine = torch.zeros_like(w, dtype=torch.bool)
        mine[1:pages + 1, 1] = True
        mine[pages, 1, N - (pages - 1) * page:] = False
        assert torch.all(w[~mine] == -3.0) and torch.all(pos[~mine] == -9) and torch.all(w[mine] >= 0)
        return pos[mine]

    lse = torch.full((1, H, N), 20.0, device="cuda")
    assert torch.equal(check(lambda w, pos: B.twist_attn_core_weights(B.attn_core_weights_args(
        B.BF16, 1, 1, N, H, KV, D, 6, 3, qkv=x, lse=lse, page_table=table, weights=w, slot_pos=pos, **heads))), torch.arange(N, dtype=torch.int32, device="cuda"))
    check(lambda w, pos: B.twist_attn_weights(B.attn_weights_args(
        B.BF16, 1, 1, H, KV, D, 6, 3, q=x[:, :1, :H * D], lse=lse[:, :, :1].contiguous(), k_cache=k, page_table=table, kv_len=i32([[N]]), new_len=i32([[N]]),
        weights=w, slot_pos=pos, **heads)))
