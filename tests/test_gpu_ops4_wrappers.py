"""What the Python wrappers of the rotation and the 4-bit cache refuse on the device: each of a call's
tensors of a wrong type, shape or layout (nothing is launched)."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def nv():
    import paper_2312_04429_amd as P
    return P


def i32(*shape):
    return torch.zeros(*shape, dtype=torch.int32, device="cuda")


@pytest.fixture
def args():
    x = torch.zeros(2, 3, 128, dtype=torch.float16, device="cuda")
    return x, list(nv().nv_kv4_pages(4, 2, 64, "cuda")), i32(2, 2), i32(2)


def wrong(t):
    """Tensors that may not stand for t: type, size, strides, device."""
    yield t.view(torch.uint8).to(torch.float64)
    yield t[:1]
    yield t.cpu()
    if t.dim() > 1:
        yield t.transpose(0, 1)


def test_pages_are_checked_one_by_one(args):
    x, pages, table, n = args
    for i in range(4):
        for bad in wrong(pages[i].view(torch.uint8)):
            p = list(pages)
            p[i] = bad
            for call in (lambda: nv().nv_op_kv4_append(x, x, p, table, n),
                         lambda: nv().nv_op_kv4_read(p, table, n, 3),
                         lambda: nv().nv_op_attention_kv4(x, p, table, n, 1.0)):
                with pytest.raises((ValueError, RuntimeError)):
                    call()
    nv().nv_op_attention_kv4(x, pages, table, n, 1.0)


def test_other_tensors_of_the_cache(args):
    x, pages, table, n = args
    P = nv()
    for bad in (n.long(), i32(3), n.cpu(), i32(4)[::2]):
        for call in (lambda: P.nv_op_kv4_append(x, x, pages, table, bad),
                     lambda: P.nv_op_kv4_append(x, x, pages, table, n, bad),
                     lambda: P.nv_op_kv4_read(pages, table, bad, 3),
                     lambda: P.nv_op_kv4_read(pages, table, n, 3, bad),
                     lambda: P.nv_op_attention_kv4(x, pages, table, bad, 1.0),
                     lambda: P.nv_op_attention_kv4(x, pages, table, n, 1.0, qpos=bad)):
            with pytest.raises(ValueError):
                call()
    for bad in (table.long(), i32(3, 2), i32(2, 4)[:, ::2], i32(4)):
        with pytest.raises(ValueError):
            P.nv_op_kv4_append(x, x, pages, bad, n)
        with pytest.raises(ValueError):
            P.nv_op_attention_kv4(x, pages, bad, n, 1.0)
    for k, v in ((x, x.bfloat16()), (x, x[:, :2]), (x.float(), x.float()), (x[..., :64], x[..., :64]),
                 (x[..., ::2], x[..., ::2]), (x, x.cpu())):
        with pytest.raises(ValueError):
            P.nv_op_kv4_append(k, v, pages, table, n)
    for out in ((x, x.bfloat16()), (x[:, :2], x), (x[:1], x)):
        with pytest.raises(ValueError):
            P.nv_op_kv4_read(pages, table, n, 3, out=out)
    with pytest.raises(ValueError):
        P.nv_op_kv4_read(pages, table, n, 3, dtype=torch.int32)
    with pytest.raises(P._native.NvError):
        P.nv_op_attention_kv4(x, pages, table, n, float("nan"))


def test_rope_tensors():
    P = nv()
    x, f, w = torch.zeros(2, 3, 128, dtype=torch.float16, device="cuda"), P.nv_rope_freqs((64,)), \
        torch.ones(64, device="cuda")
    ok = dict(q=x, k=x, dh=64, pos=i32(2, 3, 1), axes=(64,), freqs=f, q_weight=w, k_weight=w)
    P.nv_op_qk_rope(**ok)
    for bad in (dict(q=x.float()), dict(q=x[0]), dict(q=x[..., ::2]), dict(k=x.bfloat16()), dict(k=x[:, :2]),
                dict(k=x[..., :100]), dict(dh=60), dict(dh=0), dict(pos=i32(2, 3, 2)), dict(pos=i32(2, 3)),
                dict(pos=i32(2, 3, 1).long()), dict(axes=(32,)), dict(freqs=f.float()), dict(freqs=f.cpu()),
                dict(q_weight=w.half()), dict(k_weight=w[:32]), dict(eps=None), dict(out=(x, x[:, :2])),
                dict(out=(x.bfloat16(), x)), dict(axes=(32, 32), pos=i32(2, 2, 3).transpose(1, 2))):
        with pytest.raises(ValueError):
            P.nv_op_qk_rope(**{**ok, **bad})
    for bad in (dict(eps=-1.0), dict(halves=2), dict(axes=(2,) * 32, pos=i32(2, 3, 32)),
                dict(axes=(63, 1), pos=i32(2, 3, 2))):
        with pytest.raises(P._native.NvError):
            P.nv_op_qk_rope(**{**ok, **bad})
