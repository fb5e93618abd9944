"""A stored int8 layer whose tensors are not what the products read is refused before its addresses reach a kernel."""

import copy

import pytest
import torch

import paper_2410_16135_amd as vnm
from paper_2410_16135_amd import binding

OUT, INN, V, M = 128, 256, 64, 8


def layer(device="cpu"):
    s = vnm.vnm_query_sizes(OUT, INN, V, M)
    c = vnm.CompressedI8(torch.zeros(s.values_elems, dtype=torch.int8, device=device),
                         torch.full((s.meta_bytes,), 0x44, dtype=torch.uint8, device=device),
                         torch.arange(4, dtype=torch.uint8, device=device).repeat(s.row_blocks * s.col_blocks), None,
                         torch.ones(OUT, device=device), OUT, INN, V, M)
    c.packed = torch.zeros(binding._i8_packed_bytes(c, 2), dtype=torch.uint8, device=device)
    return c


# field -> what is put in its place
WRONG = [
    ("scale", lambda t: t.half()), ("scale", lambda t: t[:-1]), ("scale", lambda t: t[:1].expand(OUT)), ("scale", lambda t: t.double()),
    ("scale", lambda t: torch.ones(2 * OUT, device=t.device)[::2]),
    ("meta", lambda t: t[:-1]), ("meta", lambda t: t.float()), ("meta", lambda t: t[:1].expand(t.numel())),
    ("colidx", lambda t: t[4:]), ("colidx", lambda t: t.int()), ("values", lambda t: t[:-2]), ("values", lambda t: t.half()),
    ("packed", lambda t: t[:-1]), ("packed", lambda t: t[:1].expand(t.numel())), ("packed", lambda t: t[:t.numel() // 4].float()),
    ("out", lambda n: n + 64), ("inn", lambda n: n + 64), ("M", lambda n: 4), ("V", lambda n: 128 if n == 64 else 64),
]


# (one row block of 128 rows needs fewer columns than two of 64, so V too shows in the sizes)
@pytest.mark.parametrize("name,wrong", WRONG, ids=["%s-%d" % (w[0], i) for i, w in enumerate(WRONG)])
def test_a_layer_of_other_tensors_is_refused(name, wrong):
    c = layer()
    binding._check_layer_i8(c, 2)
    setattr(c, name, wrong(getattr(c, name)))
    assert not c.checked                                     # a field was assigned: the next call looks again
    with pytest.raises(AssertionError):
        binding._check_layer_i8(c, 2)


def test_a_layer_is_looked_at_once():
    c = layer()
    assert not c.checked
    binding._check_layer_i8(c, 2)
    assert c.checked and copy.copy(c).checked
    c.scale = c.scale.clone()
    assert not c.checked
    binding._check_layer_i8(c, 2)
    c.packed = None                                          # (the kernel on the triple then serves it)
    binding._check_layer_i8(c, 2)
    assert c.checked


@pytest.mark.gpu
@pytest.mark.parametrize("name,wrong", WRONG + [("scale", lambda t: t.cpu()), ("meta", lambda t: t.cpu()), ("packed", lambda t: t.cpu())])
def test_the_products_refuse_it(name, wrong):
    c = layer("cuda:0")
    q, s = torch.zeros(200, INN, dtype=torch.int8, device="cuda:0"), torch.ones(200, device="cuda:0")
    staged = vnm.vnm_stage_q(q, M)
    assert bool((vnm.vnm_spmm_i8(q, s, c) == 0).all()) and bool((vnm.vnm_spmm_i8_staged(staged, s, c) == 0).all())
    setattr(c, name, wrong(getattr(c, name)))
    for call in (lambda: vnm.vnm_spmm_i8(q, s, c), lambda: vnm.vnm_spmm_i8_staged(staged, s, c)):
        with pytest.raises(AssertionError):
            call()


PACKED = [lambda t: t[:-1], lambda t: t[:1].expand(t.numel()), lambda t: t.float(), lambda t: t.view(torch.int8), lambda t: t.repeat(2)[::2]]


@pytest.mark.parametrize("wrong", PACKED)
def test_packing_refuses_other_memory(wrong, monkeypatch):
    """Memory that is not whole bytes one after the other is not packed into, however many elements it has; nothing is allocated
    to find out."""
    launched = []
    monkeypatch.setattr(binding, "_check_triple", lambda *a: None)
    monkeypatch.setattr(binding, "_launch", lambda *a: launched.append(a))
    monkeypatch.setattr(binding, "_i8_packed", lambda *a: pytest.fail("memory for a layer that has some"))
    c = layer()
    vnm.vnm_pack_i8(c)
    assert len(launched) == 1
    c.packed = wrong(c.packed)
    with pytest.raises(AssertionError):
        vnm.vnm_pack_i8(c)
    assert len(launched) == 1


@pytest.mark.gpu
def test_packing_on_the_device():
    c = layer("cuda:0")
    for wrong in PACKED + [lambda t: t.cpu()]:
        d = copy.copy(c)
        d.packed = wrong(c.packed)
        with pytest.raises(AssertionError):
            vnm.vnm_pack_i8(d)
    before = torch.cuda.memory_allocated()
    torch.cuda.reset_peak_memory_stats()
    vnm.vnm_pack_i8(c)
    assert torch.cuda.max_memory_allocated() == before
