"""What the binding refuses before a call reaches the library, and the library's refusals that need no device."""
import ctypes

import pytest
import torch

import paper_2601_19404_b200 as rpo
from paper_2601_19404_b200 import binding


def _kv(dtype=torch.bfloat16, hkv=2, blocks=4, dh=64, n=3, stride=2):
    return rpo.PagedKV(torch.zeros(hkv, blocks, 16, dh, dtype=dtype), torch.zeros(hkv, blocks, 16, dh, dtype=dtype),
                       torch.zeros(n, stride, dtype=torch.int32), torch.zeros(n, dtype=torch.int32))


def _ctx(dtype=1):
    """A context without a handle: every call that gets through the binding is refused by the library (NULL context)."""
    c = rpo.Context.__new__(rpo.Context)
    c.lib, c.shape, c.handle = rpo.load_library(), rpo.shape_preset("tiny", dtype=dtype), ctypes.c_void_p()
    return c


def test_the_cache_description():
    kv = _kv()
    assert (kv.struct.n_blocks, kv.struct.n_seqs, kv.struct.table_stride, kv.struct.n_kv_heads, kv.struct.head_dim) == (4, 3, 2, 2, 64)
    k, t, n = torch.zeros(2, 4, 16, 64), torch.zeros(3, 2, dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
    for bad in ((k[:, :, :8], k[:, :, :8], t, n), (k, k[:1], t, n), (k, k.bfloat16(), t, n), (k, k, t.long(), n), (k, k, t, n[:2]),
                (k, k, t, n.float()), (k, k, t.t(), n), (k[0], k[0], t, n), (k.transpose(0, 1), k.transpose(0, 1), t, n),
                (k, k.transpose(0, 1).contiguous().transpose(0, 1), t, n)):
        with pytest.raises(ValueError):
            rpo.PagedKV(*bad)


def test_calls_check_types_shapes_and_layouts():
    ctx, kv = _ctx(), _kv()
    bf = torch.bfloat16
    q, off = torch.zeros(5, 4, 64, dtype=bf), torch.zeros(4, dtype=torch.int32)
    out, lse = torch.zeros_like(q), torch.zeros(5, 4)
    good = dict(d_q=q, kv=kv, d_q_offsets=off, max_chunk=2, d_out=out, d_lse_out=lse)
    with pytest.raises(rpo.RpoError):                                       # through the binding, refused: NULL context
        ctx.chunk_attention(**good)
    for change in (dict(d_q=q.float()), dict(d_q=q[..., :32]), dict(d_q=q.transpose(0, 1)), dict(d_q=torch.zeros(5, 64, 4, dtype=bf).transpose(1, 2)),
                   dict(d_q_offsets=off[:3]), dict(d_q_offsets=off.long()), dict(d_out=out.float()), dict(d_out=out[:4]), dict(d_lse_out=lse[:, :3]),
                   dict(d_lse_out=lse.double()), dict(d_k_new=torch.zeros(5, 2, 64, dtype=bf)),
                   dict(d_k_new=torch.zeros(4, 2, 64, dtype=bf), d_v_new=torch.zeros(4, 2, 64, dtype=bf)),
                   dict(d_k_new=torch.zeros(5, 2, 64, dtype=bf), d_v_new=torch.zeros(5, 4, 64, dtype=bf)[:, :2]), dict(kv=_kv(torch.float32)),
                   dict(kv=_kv(torch.float16))):
        with pytest.raises(ValueError):
            ctx.chunk_attention(**{**good, **change})
    mass = torch.zeros(3, 2, 40)
    good = dict(d_q=q, kv=kv, d_q_offsets=off, max_chunk=2, d_lse=lse, d_mass_out=mass)
    with pytest.raises(rpo.RpoError):
        ctx.attention_mass(**good)
    for change in (dict(d_lse=lse[:4]), dict(d_mass_out=mass[:2]), dict(d_mass_in=mass[..., :30]), dict(d_mass_out=mass.double()), dict(d_q=q.float())):
        with pytest.raises(ValueError):
            ctx.attention_mass(**{**good, **change})
    pos, src, lens = torch.zeros(3, 2, 40, dtype=torch.int32), torch.zeros(3, 2, 8, dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
    good = dict(kv=kv, d_mass=mass, d_positions=pos, budget=8, d_lens_out=lens, d_src_out=src, d_mass_out=mass, d_positions_out=pos)
    with pytest.raises(rpo.RpoError):
        ctx.evict_cache(**good)
    for change in (dict(budget=9), dict(d_positions=pos.long()), dict(d_mass=mass[..., :30]), dict(d_lens_out=lens[:2]), dict(d_positions_out=pos[..., :9]),
                   dict(d_src_out=src.long()), dict(kv=_kv(torch.float32))):
        with pytest.raises(ValueError):
            ctx.evict_cache(**{**good, **change})


def test_row_strides_of_a_fused_projection_pass():
    x = torch.zeros(6, 8, 64)
    assert binding._head_rows(x[:, :4], "q", torch.float32, 4, 64, x.device) == 512
    assert binding._head_rows(x[:1, :4], "q", torch.float32, 4, 64, x.device) == 256


def test_tensors_of_another_device_are_refused():
    """A host pointer must not reach a kernel: the device of every tensor is compared with the cache's, the cache's with the context's."""
    ctx, kv = _ctx(), _kv()
    q, off = torch.zeros(5, 4, 64, dtype=torch.bfloat16), torch.zeros(4, dtype=torch.int32)
    ctx.device = torch.device("cuda", 0)
    with pytest.raises(ValueError):
        ctx.chunk_attention(q, kv, off, 2, q.clone())
    ctx.device = None
    kv.device = torch.device("cuda", 0)
    with pytest.raises(ValueError):
        ctx.chunk_attention(q, kv, off, 2, q.clone())
    with pytest.raises(ValueError):
        ctx.attention_mass(q, kv, off, 2, torch.zeros(5, 4), torch.zeros(3, 2, 40))
