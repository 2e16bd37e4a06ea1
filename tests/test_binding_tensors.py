"""CPU: what the binding looks at before it keeps a tensor's address: a struct of addresses cannot say a tensor's type, size or strides, and
reading one as another is memory that is not the tensor's."""
import pytest

torch = pytest.importorskip("torch")

import paper_2104_05343_amd as opt   # noqa: E402


def _refused(code, make, *args, **kw):
    with pytest.raises(opt.OptimusError) as e:
        make(*args, **kw)
    assert e.value.code == code, e.value


def test_attention_bias():
    docs, prefix, table, slopes = torch.zeros(2, 8, dtype=torch.int32), torch.zeros(2, dtype=torch.int32), torch.zeros(4, 32), torch.zeros(4)
    b = opt.make_attention_bias(table=table, buckets=32, max_distance=128, documents=docs, prefix=prefix)
    assert (b.table, b.documents, b.prefix) == (table.data_ptr(), docs.data_ptr(), prefix.data_ptr())
    assert opt.make_attention_bias(slopes=slopes).slopes == slopes.data_ptr() and opt.make_attention_bias(documents=4096).documents == 4096
    assert opt.make_attention_bias(documents=torch.zeros(2, 16, dtype=torch.int32)[1]).documents
    for kw in (dict(documents=docs.long()), dict(documents=docs.to(torch.uint8)), dict(prefix=prefix.long()), dict(table=table.double()),
               dict(table=table.bfloat16()), dict(slopes=slopes.half())):
        _refused(opt.EDTYPE, opt.make_attention_bias, **kw)
    for kw in (dict(documents=torch.zeros(2, 16, dtype=torch.int32)[:, :8]), dict(documents=docs[:1].expand(2, 8)), dict(table=torch.zeros(32, 4).t()),
               dict(slopes=torch.zeros(8)[::2])):
        _refused(opt.EINVAL, opt.make_attention_bias, **kw)


def _entry(shape=(20, 30), eight=False, **kw):
    n = 1
    for k in shape:
        n *= k
    e = dict(param=torch.zeros(shape), grad=torch.zeros(shape), m=torch.zeros(shape), v=torch.zeros(shape))
    if eight:
        e.update(m=torch.zeros(n, dtype=torch.uint8), v=torch.zeros(n, dtype=torch.uint8), m_scale=torch.zeros(-(-n // 128), dtype=torch.uint8),
                 v_scale=torch.zeros(-(-n // 128), dtype=torch.uint8))
    e.update(kw)
    return e


def test_adamw_tensors_that_are_taken():
    flat = torch.zeros(4000)
    for e in (_entry(), _entry(eight=True), _entry(param=torch.zeros(20, 30, dtype=torch.bfloat16), master=torch.zeros(600)),
              _entry(grad=torch.zeros(20, 30, dtype=torch.bfloat16)), _entry(m=flat[3:603], v=flat[700:]),
              _entry(grad=torch.zeros(3, 600), grad_parts=3), _entry(n=500, m=torch.zeros(500), v=torch.zeros(500)),
              _entry(eight=True, m=torch.zeros(600, dtype=torch.float8_e4m3fn), m_scale=torch.zeros(5, dtype=torch.float8_e8m0fnu)),
              # a transposed weight whose gradient and moments lie as it does, or flat
              dict(param=torch.zeros(30, 20).t(), grad=torch.zeros(30, 20).t(), m=torch.zeros(30, 20).t(), v=torch.zeros(600))):
        a = opt.make_adamw_tensors([e])[0]
        assert (a.param, a.grad, a.m, a.v) == tuple(e[k].data_ptr() for k in ("param", "grad", "m", "v")) and a.n == e.get("n", 600)
    assert opt.make_adamw_tensors([_entry(m=4096, v=8192)])[0].m == 4096


@pytest.mark.parametrize("change", [
    dict(m=torch.zeros(600, dtype=torch.bfloat16)), dict(v=torch.zeros(600, dtype=torch.bfloat16)), dict(m=torch.zeros(600, dtype=torch.uint8)),
    dict(master=torch.zeros(600, dtype=torch.bfloat16)), dict(param=torch.zeros(600, dtype=torch.float16)), dict(grad=torch.zeros(600, dtype=torch.float64)),
    dict(eight=True, m=torch.zeros(600)), dict(eight=True, v=torch.zeros(600, dtype=torch.float8_e5m2)), dict(eight=True, m_scale=torch.zeros(5))])
def test_adamw_types(change):
    _refused(opt.EDTYPE, opt.make_adamw_tensors, [_entry(), _entry(**change)])


@pytest.mark.parametrize("change", [
    dict(m=torch.zeros(599)), dict(v=torch.zeros(1)), dict(grad=torch.zeros(599)), dict(grad_parts=2), dict(n=601), dict(master=torch.zeros(0)),
    dict(eight=True, m_scale=torch.zeros(4, dtype=torch.uint8)), dict(eight=True, v_scale=torch.zeros(1, dtype=torch.uint8))])
def test_adamw_sizes(change):
    _refused(opt.ESHAPE, opt.make_adamw_tensors, [_entry(**change)])


@pytest.mark.parametrize("change", [
    dict(param=torch.zeros(20, 60)[:, :30]), dict(grad=torch.zeros(30, 20).t()), dict(param=torch.zeros(30, 20).t()), dict(m=torch.zeros(1200)[::2]),
    dict(grad=torch.zeros(1).expand(20, 30)), dict(v=torch.zeros(20, 30, device="meta")),
    dict(eight=True, m_scale=torch.zeros(10, dtype=torch.uint8)[::2])])
def test_adamw_places(change):
    _refused(opt.EINVAL, opt.make_adamw_tensors, [_entry(**change)])


def test_adamw_state():
    f, u, s = torch.zeros(1024), torch.zeros(1024, dtype=torch.uint8), torch.zeros(8, dtype=torch.uint8)
    assert opt.make_adamw_state(f, f, master=f).m == f.data_ptr() and opt.make_adamw_state(u, u, s, s).v_scale == s.data_ptr()
    for args, kw in (((f.bfloat16(), f), {}), ((f, u), {}), ((f, f, s, s), {}), ((u, u, f, s), {}), ((f, f), dict(master=f.bfloat16()))):
        _refused(opt.EDTYPE, opt.make_adamw_state, *args, **kw)
    _refused(opt.EINVAL, opt.make_adamw_state, f[::2], f)
