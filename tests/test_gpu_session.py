"""DecodeSession on the GPU where its halves meet: uploaded caches, appended tokens and the choice of blocks."""
import numpy as np
import pytest
import torch

from test_gpu_cache_ops import Setup, _bf16, _check_attention, _check_select, _np

pytestmark = pytest.mark.gpu


def _bits(t):
    return t.contiguous().view(torch.int16).cpu().numpy().view(np.uint16)


def _chosen(s, sess, q, lens):
    """The session's summaries are those of its cache, its choice and its attention over the blocks the oracle's."""
    s.k, s.v = sess.k.view(torch.uint8).flatten(), sess.v.view(torch.uint8).flatten()
    rows, summary = s.batch * s.q_len, torch.zeros(s.summary_shape(), dtype=torch.bfloat16, device="cuda")
    s.vb.vatt_block_summary_fill(s.plan, s.k, s.table, s.ints(lens), summary, torch.cuda.current_stream().cuda_stream)
    k_max = s.vb.vatt_plan_index_segment(s.plan, 3) - s.vb.vatt_plan_index_segment(s.plan, 2)
    topk, cnt = torch.full((rows, s.hq, k_max), -9, dtype=torch.int32, device="cuda"), s.ints([[-9] * s.hq] * rows)
    sess.blocks.fill_(-9)
    sess.select_blocks(q, topk, cnt)
    sess.block_decode(q)
    torch.cuda.synchronize()
    _check_select(s, q, summary, lens, (sess.blocks, sess.block_count, topk, cnt))
    blocks, count, lists = sess.blocks.cpu().numpy(), sess.block_count.cpu().numpy(), []
    for r in range(rows):
        n = max(lens[r // s.q_len] - (s.q_len - 1 - r % s.q_len), 1)
        lists.append([np.concatenate([np.arange(j * s.block, min(j * s.block + s.block, n)) for j in blocks[r, h, :count[r, h]]]) for h in range(s.hkv)])
    _check_attention(s, q, lens, lists, sess.out_o, sess.out_lse)
    return topk, cnt


@pytest.mark.parametrize("page", [0, 32])
def test_blocks_of_an_uploaded_cache_and_of_appended_tokens(page):
    from paper_2510_05688_amd.session import DecodeSession
    s = Setup(2, 8, 2, 128, 700, page, 0, 32, seed=31, topk_frac=0.2)
    sess = DecodeSession(s.params, block_tokens=32)
    lens = [690, 333]
    q = _bf16(s.rng.normal(size=(2, 8, 128)))
    table = s.table.cpu().numpy() if page else None
    sess.upload(_bits(q), _bits(s.k.view(torch.bfloat16)), _bits(s.v.view(torch.bfloat16)), lens, [1, 2], table)
    assert sess.summary is None
    sess.fill_summary()
    _chosen(s, sess, q, lens)
    big = _bf16(np.full((2, 2, 128), 30.0))  # tokens that change which blocks are best, once they are behind the window
    for i in range(9):
        sess.append_device(big if i == 0 else _bf16(s.rng.normal(size=(2, 2, 128))), _bf16(s.rng.normal(size=(2, 2, 128))))
    lens = [699, 342]
    assert sess.seq_lens.tolist() == lens
    _chosen(s, sess, q, lens)


def test_blocks_of_tokens_appended_beside_a_random_cache():
    from paper_2510_05688_amd.session import DecodeSession
    s = Setup(2, 8, 2, 128, 500, 0, 0, 16, seed=32, topk_frac=0.2)
    sess = DecodeSession(s.params, block_tokens=16, rotary=dict(theta=10000.0)).make_cache()
    x = _bf16(s.rng.normal(size=(2, 490, 2, 128)))
    sess.write(None, x, x, s.ints([490, 200]))
    sess.make_random_cache([5, 6])
    rows = [_bf16(s.rng.normal(size=(2, 2, 128)) * (9 if i == 3 else 1)) for i in range(20)]
    for r in rows:  # (the first sequence is full after ten)
        sess.append_device_cached(r, r)
    assert sess.seq_lens.tolist() == [500, 220]
    _chosen(s, sess, _bf16(s.rng.normal(size=(2, 8, 128))), [500, 220])
    for b, n in ((0, 490), (1, 200)):  # as they are, whatever the plan's rotation
        for i, r in enumerate(rows[:10]):
            assert np.array_equal(s.rows(s.k, b, 1, [n + i])[0], _np(r[b, 1])) and np.array_equal(s.rows(s.v, b, 1, [n + i])[0], _np(r[b, 1]))


@pytest.mark.parametrize("page", [0, 32])
def test_chosen_tokens_through_the_verified_step(page):
    """Choice -> step with that top-k set: with an epsilon that asks for every token the estimate is dense attention."""
    from paper_2510_05688_amd.session import DecodeSession
    s = Setup(2, 8, 2, 128, 700, page, 0, 32, seed=33, topk_frac=0.2, epsilon=1e-4)
    sess = DecodeSession(s.params, block_tokens=32, rotary=dict(theta=10000.0)).make_cache(s.table.cpu().numpy() if page else None)
    x = [_bf16(s.rng.normal(size=(2, 691, h, 128))) for h in (8, 2, 2)]
    sess.write(*[t[:, :690].contiguous() for t in x], s.ints([690, 333]))
    q, lens = sess.write(*[t[:, 690:].contiguous() for t in x]), [691, 334]
    topk, cnt = _chosen(s, sess, q, lens)
    sess.set_seeds([7, 8])
    sess.decode_given_topk(topk, cnt, q=q)
    torch.cuda.synchronize()
    counts = sess.out_counts.cpu().numpy()
    assert (counts[..., 2] == cnt.cpu().numpy()).all() and (counts[..., 4] == counts[..., 5]).all()  # the budget is the whole residual
    _check_attention(s, q, lens, [[np.arange(n)] * 2 for n in lens], sess.out_o, sess.out_lse)
