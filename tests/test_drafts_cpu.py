"""What the binding refuses of the calls with drafted tokens and shared pages before one reaches the library, and the library's
refusals that need no device."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2601_19404_b200 as rpo

I32 = torch.int32


def _ctx(dtype=1):
    """A context without a handle: every call that gets through the binding is refused by the library (NULL context)."""
    c = rpo.Context.__new__(rpo.Context)
    c.lib, c.shape, c.handle = rpo.load_library(), rpo.shape_preset("tiny", dtype=dtype), ctypes.c_void_p()
    return c


def _cache(dtype=torch.bfloat16, n=3, stride=2, blocks=4, layers=2, hkv=2, dh=64):
    table, lens = torch.zeros(n, stride, dtype=I32), torch.zeros(n, dtype=I32)
    kv = [rpo.PagedKV(torch.zeros(hkv, blocks, 16, dh, dtype=dtype), torch.zeros(hkv, blocks, 16, dh, dtype=dtype), table, lens) for _ in range(layers)]
    return table, lens, kv


def _refused(call, good, changes):
    with pytest.raises(rpo.RpoError):                                       # through the binding, refused: NULL context
        call(**good)
    for change in changes:
        with pytest.raises(ValueError):
            call(**{**good, **change})


def test_tree_attention_checks_its_arguments():
    ctx, (_, _, layers) = _ctx(), _cache()
    q, off, parents = torch.zeros(5, 4, 64, dtype=torch.bfloat16), torch.zeros(4, dtype=I32), torch.zeros(5, dtype=I32)
    out, lse = torch.zeros_like(q), torch.zeros(5, 4)
    _refused(ctx.tree_attention, dict(d_q=q, kv=layers[0], d_q_offsets=off, d_parents=parents, max_nodes=3, d_out=out, d_lse_out=lse),
             [dict(d_parents=parents[:4]), dict(d_parents=parents.long()), dict(d_q=q.float()), dict(d_out=out[:4]), dict(d_lse_out=lse[:, :3]),
              dict(d_q_offsets=off[:3]), dict(d_k_new=torch.zeros(5, 2, 64, dtype=torch.bfloat16)), dict(kv=_cache(torch.float32)[2][0])])


def test_verification_checks_its_arguments():
    ctx, rows, vocab, n = _ctx(), 6, 10, 2
    z, ints = torch.zeros(rows, vocab), torch.zeros(rows, dtype=I32)
    path, one, logp = torch.zeros(n, 4, dtype=I32), torch.zeros(n, dtype=I32), torch.zeros(n, 4)
    good = dict(d_logits=z, d_tokens=ints, d_parents=ints, d_offsets=torch.zeros(n + 1, dtype=I32), d_uniform=torch.zeros(rows), sampler=rpo.Sampler(), d_path_out=path,
                d_n_path_out=one, d_next_out=one, d_logprobs_out=logp, d_draft_probs=z)
    _refused(ctx.verify_drafts, good,
             [dict(d_logits=z.double()), dict(d_logits=z.t()), dict(d_logits=torch.zeros(rows, vocab, 2)[..., 0]), dict(d_draft_probs=z[:, :9]), dict(d_draft_probs=z.half()),
              dict(d_tokens=ints[:5]), dict(d_parents=ints.long()), dict(d_uniform=torch.zeros(rows).double()), dict(d_offsets=torch.zeros(n, dtype=I32)),
              dict(d_offsets=torch.zeros(0, dtype=I32)), dict(d_n_path_out=one[:1]), dict(d_next_out=one.long()), dict(d_logprobs_out=logp[:, :3])])
    with pytest.raises(rpo.RpoError):
        ctx.verify_drafts(**{**good, "d_logits": torch.zeros(rows, 12)[:, :vocab], "d_draft_probs": None, "d_logprobs_out": None})      # strided rows pass


def test_calls_without_rows_pass_whatever_their_strides():
    """Tensors without elements may have any strides: those that come from numpy have zeros."""
    ctx, n, vocab = _ctx(0), 2, 10
    (_, _, layers), none = _cache(torch.float32, n=n), torch.from_numpy(np.zeros((0, vocab), dtype=np.float32))
    rows = torch.from_numpy(np.zeros((0, 4, 64), dtype=np.float32))
    assert none.stride() == (0, 0) and rows.stride() == (0, 0, 0)
    ints, off, one = torch.zeros(0, dtype=I32), torch.zeros(n + 1, dtype=I32), torch.zeros(n, dtype=I32)
    with pytest.raises(rpo.RpoError):                                       # through the binding, refused: NULL context
        ctx.verify_drafts(none, ints, ints, off, torch.zeros(0), rpo.Sampler(), torch.zeros(n, 4, dtype=I32), one, one, d_draft_probs=none)
    with pytest.raises(rpo.RpoError):
        ctx.tree_attention(rows, layers[0], off, ints, 3, torch.zeros(0, 4, 64))


def test_layers_and_pools_check_their_tensors():
    table, lens, layers = _cache()
    assert rpo.PagedLayers(layers).n_seqs == 3
    for bad in ([], [layers[0], _cache()[2][0]], [layers[0], _cache(torch.float32)[2][0]],
                [layers[0], rpo.PagedKV(torch.zeros(2, 5, 16, 64, dtype=torch.bfloat16), torch.zeros(2, 5, 16, 64, dtype=torch.bfloat16), table, lens)],
                [layers[0], rpo.PagedKV(layers[0].d_k, layers[0].d_v, table, lens.clone())]):
        with pytest.raises(ValueError):
            rpo.PagedLayers(bad)
    refs, one, held = torch.zeros(4, dtype=I32), torch.zeros(1, dtype=I32), torch.zeros(3, dtype=I32)
    assert rpo.PagePool(refs, refs.clone(), one, table, held).struct.n_blocks == 4
    for bad in ((refs[:3], refs, one, table, held), (refs, refs.long(), one, table, held), (refs, refs, refs, table, held), (refs, refs, one, table.long(), held),
                (refs, refs, one, table.t(), held), (refs, refs, one, table, held[:2])):
        with pytest.raises(ValueError):
            rpo.PagePool(*bad)
    pool = rpo.PagePool.empty(5, 3, 2, device="cpu")
    assert pool.d_free.tolist() == [4, 3, 2, 1, 0] and int(pool.d_n_free) == 5 and pool.d_held.tolist() == [0, 0, 0] and (pool.d_block_table == -1).all()


def test_page_calls_check_their_arguments():
    ctx, (table, lens, kv) = _ctx(), _cache()
    layers, refs = rpo.PagedLayers(kv), torch.zeros(4, dtype=I32)
    pool = rpo.PagePool(refs, refs.clone(), torch.zeros(1, dtype=I32), table, torch.zeros(3, dtype=I32))
    other = rpo.PagePool.empty(4, 3, 2, device="cpu")
    ints, off, path = torch.zeros(2, dtype=I32), torch.zeros(4, dtype=I32), torch.zeros(3, 5, dtype=I32)
    wrong = rpo.PagedLayers(_cache(torch.float32)[2])
    _refused(ctx.fork_pages, dict(pool=pool, layers=layers, d_src=ints, d_dst=ints, d_fork_lens=ints, d_lens_out=lens),
             [dict(d_dst=ints[:1]), dict(d_fork_lens=ints.long()), dict(d_lens_out=lens[:2]), dict(pool=other), dict(layers=wrong)])
    _refused(ctx.reserve_pages, dict(pool=pool, layers=layers, d_lens=lens, d_target_lens=lens),
             [dict(d_lens=lens[:2]), dict(d_target_lens=lens.long()), dict(pool=other), dict(layers=wrong)])
    _refused(ctx.commit_path, dict(layers=layers, d_q_offsets=off, d_path=path, d_n_path=lens, d_lens_out=lens),
             [dict(d_q_offsets=off[:3]), dict(d_path=path[:2]), dict(d_path=path.long()), dict(d_n_path=lens[:2]), dict(d_lens_out=lens.float()), dict(layers=wrong)])
    ctx.device = torch.device("cuda", 0)                                     # a host pointer must not reach a kernel
    for call in (lambda: ctx.reserve_pages(pool, layers, lens, lens), lambda: ctx.commit_path(layers, off, path, lens, lens)):
        with pytest.raises(ValueError):
            call()
