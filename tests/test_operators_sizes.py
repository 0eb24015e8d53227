"""Sizes at the ends of 32 bits: refused, not cut."""
import ctypes as C

import pytest


def test_the_c_calls_refuse_adapter_sizes_whose_tiles_would_pass_32_bits():
    import paper_1711_09846_b200 as pbt
    from paper_1711_09846_b200.binding import PbtAdapterDesc
    lib, n = pbt.load_library(), C.c_size_t(0)

    def desc(**kw):
        d = PbtAdapterDesc()
        d.rows, d.inputs, d.outputs, d.rank, d.n_adapters, d.n_segments, d.dtype = 10, 1, 1, 1, 1, 2, kw.pop("dtype", 1)
        for name in ("weight", "A", "B", "scale", "row_offsets", "adapter_ids", "x", "y", "s", "dy", "dx", "dA", "dB", "status_device"):
            setattr(d, name, 4096)
        d.ld_weight = d.ld_x = d.ld_dx = d.ld_y = d.ld_dy = 0x7FFFFFFF
        for k, v in kw.items():
            setattr(d, k, v)
        return d
    for dtype in (0, 1):
        for size in ("rows", "inputs", "outputs", "n_segments"):
            for backward in (0, 1):
                assert lib.pbt_adapter_query_workspace(C.byref(desc(dtype=dtype, **{size: 0x7FFFFFFF})), backward, C.byref(n)) == 2, size
            assert lib.pbt_adapter_forward(C.byref(desc(dtype=dtype, **{size: 0x7FFFFFFF - 100})), 4096, 1 << 60, None) == 2, size
            assert lib.pbt_adapter_backward(C.byref(desc(dtype=dtype, **{size: 0x7FFFFFFF - 100})), 4096, 1 << 60, None) == 2, size
        assert lib.pbt_adapter_query_workspace(C.byref(desc(dtype=dtype, rows=0x7FFFFFFF - 4096)), 1, C.byref(n)) == 0


@pytest.mark.gpu
def test_the_python_calls_refuse_sizes_beyond_32_bits():
    import torch
    import paper_1711_09846_b200 as pbt
    many = 2 ** 32 + 5                                   # cut to 32 bits: 5
    bf = dict(device="cuda", dtype=torch.bfloat16)
    offsets, ids = (torch.tensor(v, dtype=torch.int32, device="cuda") for v in ([0, 5], [0]))
    one = torch.ones(1, device="cuda")
    layer = pbt.AdapterProjection(torch.ones(2, 1, **bf), torch.ones(1, 1, 1, **bf), torch.ones(1, 2, 1, **bf), one)
    long = torch.empty(many, 1, **bf)
    with pytest.raises(ValueError):
        layer.forward(long, offsets, ids)
    with pytest.raises(ValueError):
        layer.backward(long.expand(many, 2), long, torch.ones(5, 1, device="cuda"), offsets, ids)
    with pytest.raises(ValueError):
        pbt.AdapterProjection(long, torch.ones(1, 1, 1, **bf), long.view(1, many, 1), one)
    del long
    x = torch.ones(1, 1, 1, **bf)
    for shape in ((1, many, 1), (many, 1, 1), (1, 1, many)):
        with pytest.raises(ValueError):
            pbt.block_norm_forward(x.expand(shape), next_weight=torch.ones(1, 1, device="cuda").expand(shape[0], shape[2]))
    g = torch.zeros(4, device="cuda")
    for kw in (dict(groups=[2 ** 32]), dict(groups=[0], n_groups=2 ** 32 + 1), dict(groups=[-2 ** 32]), dict(groups=[2 ** 31 - 1])):
        with pytest.raises(ValueError):
            pbt.GradientClip([g], **kw)
