"""A cache whose two sides lie on different devices, or whose encoded planes are
of another type, is refused where it is made: the kernels get addresses only.
(Stand-ins for tensors: only what the checks look at.)"""
import pytest

torch = pytest.importorskip("torch")


class Fake:
    is_cuda = True

    def __init__(self, shape, dtype, device):
        self.shape, self.dtype, self.device = shape, dtype, torch.device(device)

    def dim(self):
        return len(self.shape)

    def stride(self, i=None):
        st = [1]
        for n in self.shape[:0:-1]:
            st.insert(0, st[0] * n)
        return st if i is None else st[i]

    def numel(self):
        n = 1
        for s in self.shape:
            n *= s
        return n

    def is_contiguous(self):
        return True

    def element_size(self):
        return torch.empty(0, dtype=self.dtype).element_size()

    def data_ptr(self):
        return 1 << 20


@pytest.fixture(scope="module")
def Q():
    from paper_2509_26436_gb300 import build
    build.build()
    import paper_2509_26436_gb300 as Q
    return Q


def test_sides_on_two_devices(Q):
    sides = [Fake((4, 16, 2, 64), torch.float16, f"cuda:{i}") for i in (0, 1)]
    with pytest.raises(ValueError, match="devices"):
        Q.PagedCache(*sides, 16)


def _encoded(Q, device="cuda:0", **other):
    rows, D, p = 4 * 16 * 2, 64, Q.Params(group_s=16)
    planes = dict(codes=((rows, D // 2), torch.uint8, device), flags=((rows, D // 16), torch.uint8, device),
                  scales=((rows, D // 64), torch.float16, device))
    planes.update(other)
    t = {name: Fake(*args) for name, args in planes.items()}
    return Q.Encoded(t["codes"], t["flags"], t["scales"], None, None, rows, D, p)


@pytest.mark.parametrize("other", [dict(device="cuda:1"), dict(flags=((128, 4), torch.uint8, "cuda:1")),
                                   dict(scales=((128, 1), torch.float32, "cuda:0")),
                                   dict(scales=((128, 1), torch.float16, "cuda:1")),
                                   dict(codes=((128, 32), torch.int32, "cuda:0")),
                                   dict(flags=((128, 4), torch.int64, "cuda:0"))])
@pytest.mark.parametrize("swap", [False, True])
def test_encoded_planes(Q, other, swap):
    k, v = _encoded(Q), _encoded(Q, **other)
    if swap:
        k, v = v, k
    with pytest.raises(ValueError, match="one device"):
        Q.PagedCache(k, v, 16, heads=2)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.int8, torch.uint8])
def test_planes_of_the_device_are_taken(Q, dtype):
    """Bytes are bytes: codes held as int8 go in as before."""
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    c = Q.empty_paged_cache(4, 16, 2, 64, params=Q.Params(group_s=16))
    sides = [Q.Encoded(e.codes.view(dtype), e.flags.view(dtype), e.scales, None, None, e.rows, e.K, e.params) for e in (c.k, c.v)]
    assert Q.PagedCache(*sides, 16, heads=2).num_pages == 4
