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
