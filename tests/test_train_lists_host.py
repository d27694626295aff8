"""What the binding of the operators beside the round keeps, takes and refuses, on host memory: tensors
that say they are on a device stand for device tensors, and no call here reaches the library's GPU work."""
import os
import weakref

import numpy as np
import pytest

torch = pytest.importorskip("torch")


class Device0(torch.Tensor):
    """A host tensor that says it is on device 0."""
    is_cuda = property(lambda self: True)

    def get_device(self):
        return 0


def on_device(x):
    """A Device0 over a numpy array's own memory, or a tensor's."""
    x = torch.from_numpy(x) if isinstance(x, np.ndarray) else x
    return torch.Tensor._make_subclass(Device0, x)   # with no reference to x beside its memory


@pytest.fixture(scope="module")
def E():
    from paper_2205_14473_amd import build as bld
    if bld.is_stale() and "EA_LIB" not in os.environ:
        bld.build()
    import paper_2205_14473_amd as E
    return E


def test_a_list_holds_its_gradients_memory(E):
    """The addresses in the list stay those of live memory when a gradient's storage is replaced, and until
    other gradients take their place."""
    a = [np.ones(8, np.float32) for _ in range(3)]
    memory = [weakref.ref(x) for x in a]
    g = [on_device(x) for x in a]
    del a
    at = [t.data_ptr() for t in g]
    tl = E.TensorList(g)
    g[1].data = torch.zeros(5)
    g[2].set_(torch.zeros(8))
    assert [e.g for e in tl.array] == at
    assert all(m() is not None for m in memory)
    other = [on_device(np.zeros(8, np.float32)) for _ in range(3)]
    with pytest.raises(ValueError, match="2 gradients for 3"):
        tl.set_grads(other[:2])                    # a refused replacement lets go of nothing
    assert all(m() is not None for m in memory)
    tl.set_grads(other)
    assert memory[1]() is None and memory[2]() is None


@pytest.fixture
def current_device(E, monkeypatch):
    """Device 0 is the current one, whether there is a GPU or not."""
    from paper_2205_14473_amd import _train
    _train._dtypes()
    monkeypatch.setattr(_train, "_current", lambda: 0)


def embedding(E):
    c = E.Embed(tokens=4, vocab=7, dim=6, table_stride=6, x_stride=6, padding=-1, scale=1.0, index_bits=64)
    return c, on_device(torch.zeros(4, dtype=torch.int64)), on_device(torch.zeros(4, 6)), on_device(torch.zeros(7, 6))


@pytest.mark.parametrize("plain", [True, False])
def test_a_workspace_may_be_a_raw_pointer(E, current_device, plain):
    """Beside tensors of the plain form and of others alike: the call gets as far as the library, which
    refuses the address (8 is not 16-byte aligned)."""
    c, ids, dx, dtable = embedding(E)
    if not plain:
        ids = on_device(torch.zeros(2, 2, dtype=torch.int64))
        dx = on_device(torch.zeros(2, 2, 6))
    with pytest.raises(E.EAError, match="workspace is not 16-byte aligned"):
        E.ea_embed_grad(c, ids, dx, dtable, False, 8, 0)
    tl = E.TensorList([on_device(torch.zeros(5))])
    with pytest.raises(E.EAError, match="workspace is not 8-byte aligned"):
        E.ea_grad_norm(tl, 1.0, 1.0, 16, 16, 4, 0)


def test_strides_of_one_element_do_not_matter(E):
    """A dimension of one element has no order: a convolution of 1 x 1 is laid out alike under either of
    torch's memory formats, also beside one of 3 x 3 whose format differs from the default."""
    def like(shape, strides):
        return on_device(torch.zeros(shape).as_strided(shape, strides))

    wide, narrow = ((8, 4, 3, 3), (36, 1, 12, 4)), (8, 4, 1, 1)
    for a, b in (((4, 1, 1, 1), (4, 1, 4, 4)), ((4, 1, 4, 4), (4, 1, 1, 1))):
        p, g = [like(*wide), like(narrow, a)], [like(*wide), like(narrow, b)]
        tl = E.TensorList(g, p=p)
        assert [e.p for e in tl.array] == [t.data_ptr() for t in p]
        assert [e.g for e in tl.array] == [t.data_ptr() for t in g]
        tl.set_grads([like(*wide), like(narrow, a)])
    # the order of dimensions that have one does
    with pytest.raises(ValueError, match="strides"):
        E.TensorList([like(*wide), like((8, 4, 1, 1), (1, 8, 1, 1))], p=[like(*wide), like(narrow, (4, 1, 1, 1))])


@pytest.mark.parametrize("bits,kind", [(64, torch.complex64), (32, torch.complex32), (32, torch.float32),
                                       (64, torch.float64), (64, torch.int32), (32, torch.int64)])
def test_ids_are_integers(E, current_device, bits, kind):
    """Types of an id's size that hold no integers are refused (the library would refuse the rest: a scale
    of NaN, a workspace at 8)."""
    c, _, x, table = embedding(E)
    c.index_bits, ids = bits, on_device(torch.zeros(4, dtype=kind))
    with pytest.raises(ValueError, match=f"expected {bits}-bit integers"):
        E.ea_embed_grad(c, ids, x, table, False, 8, 0)
    c.scale = float("nan")
    with pytest.raises(ValueError, match=f"expected {bits}-bit integers"):
        E.ea_embed_lookup(c, table, ids, x, 0)


@pytest.mark.parametrize("name", ["weight_decay", "lr_scale"])
def test_factors_come_one_for_all_or_one_for_each(E, name):
    g = [on_device(torch.zeros(3)) for _ in range(2)]
    for bad in ([0.1], [0.1, 0.2, 0.3], []):
        with pytest.raises(ValueError, match=f"{len(bad)} values of {name}, and 2 tensors"):
            E.TensorList(g, **{name: bad})
    for one in (0.5, 1, np.float32(0.5), torch.tensor(0.5)):
        assert [getattr(e, name) for e in E.TensorList(g, **{name: one}).array] == [float(one)] * 2
    for each in ([0.25, 0.5], (0.25, 0.5), np.array([0.25, 0.5]), torch.tensor([0.25, 0.5])):
        assert [getattr(e, name) for e in E.TensorList(g, **{name: each}).array] == [0.25, 0.5]


def test_entries_of_p_that_are_no_tensors_are_named(E):
    g = [on_device(torch.zeros(3)) for _ in range(2)]
    for bad in (None, 3):
        for at in (0, 1):
            p = [on_device(torch.zeros(3)) for _ in range(2)]
            p[at] = bad
            with pytest.raises(ValueError, match=rf"p\[{at}\]: expected a tensor, got {type(bad).__name__}"):
                E.TensorList(g, p=p)
