"""Arguments that the operators which run and score a quantized model refuse, on the
CPU: the Python entries with a library that only notes its calls, and the C entries
before any CUDA work."""
import pytest

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def jarq():
    from paper_2609_38599_gb300 import jarq as mod
    return mod


class FakeCuda:
    """What the Python entries ask of a CUDA tensor."""

    __module__ = "torch.fake"
    is_cuda, device = True, "cuda:0"

    def __init__(self, shape, dtype, contiguous=True):
        self.shape, self.dtype, self._contiguous = torch.Size(shape), dtype, contiguous

    def is_contiguous(self):
        return self._contiguous

    def data_ptr(self):
        return 0x1000

    def get_device(self):
        return 0

    def stride(self):
        return (self.shape[1], 1)

    def __getitem__(self, _):
        return self


@pytest.fixture
def calls(jarq, monkeypatch):
    """The C calls that an entry makes: (name, arguments)."""
    made = []

    class Library:
        jarq_status_string = staticmethod(lambda status: b"status")

        def __getattr__(self, name):
            return lambda *a: made.append((name, a)) or 0

    T = jarq._torch()
    monkeypatch.setattr(jarq, "_lib", Library())
    monkeypatch.setattr(T, "empty", lambda shape, dtype, device: FakeCuda(shape, dtype))
    monkeypatch.setattr(T, "stream", lambda index: 0)
    return made


def codes(dout=6, din=256, g=64, zrows=None, zcols=None, qdtype=torch.uint8, zdtype=torch.int32, contiguous=True):
    zcols = din // g if zcols is None else zcols
    return FakeCuda((dout, din), qdtype, contiguous), FakeCuda((dout if zrows is None else zrows, zcols), zdtype), g, 3


def test_integer_codes_of_matching_shapes_are_made(jarq, calls):
    flat = codes()
    flat[1].shape = torch.Size((24,))
    for args in (codes(), codes(din=30, g=10), codes(dout=1, din=64, g=64), flat):
        jarq.integer_codes(*args)
        (name, a), = calls
        assert name == "jarq_integer_codes" and a[2:6] == (*args[0].shape, args[2], 3)
        calls.clear()


# zero points of another group size, layer or type: the kernel would read past them
@pytest.mark.parametrize("args", [codes(g=32, zcols=4), codes(zcols=1), codes(zcols=5), codes(zrows=5), codes(zrows=0),
                                  codes(zdtype=torch.int64), codes(qdtype=torch.int8), codes(contiguous=False)])
def test_integer_codes_of_other_shapes_are_refused(jarq, calls, args):
    with pytest.raises(TypeError):
        jarq.integer_codes(*args)
    assert not calls


def test_integer_codes_wants_matrices_of_the_device(jarq, calls):
    q, z, g, bits = codes()
    for bad in (FakeCuda((6, 2, 128), torch.uint8), torch.zeros(6, 256, dtype=torch.uint8)):
        with pytest.raises(TypeError):
            jarq.integer_codes(bad, z, g, bits)
    with pytest.raises(TypeError):
        jarq.integer_codes(q, torch.zeros(6, 4, dtype=torch.int32), g, bits)
    with pytest.raises(TypeError):
        jarq.integer_codes(q, FakeCuda((23,), torch.int32), g, bits)
    for wrong in (0, -64, 48, 512):
        with pytest.raises(jarq.JarqError) as e:
            jarq.integer_codes(q, z, wrong, bits)
        assert e.value.status == jarq.JARQ_ERR_ARG
    assert not calls


F16, MOST = 1, 2 ** 31 - 4096


# sizes past which the kernels' 32-bit indexes would wrap; an empty batch is checked
# like any other, and does no CUDA work
@pytest.mark.parametrize("n,d", [(2 ** 31 - 1, 64), (MOST + 1, 64), (0, MOST + 1), (0, 2 ** 31 - 1), (1, MOST)])
def test_rows_to_quantize_stay_within_the_indexes(jarq, n, d):
    L = jarq.library()
    assert L.jarq_quantize_rows(None, F16, n, d, d, None, d, None, None) == jarq.JARQ_ERR_ARG


def test_layers_stay_within_the_indexes(jarq):
    L = jarq.library()

    def layer(n, dout):
        return {L.jarq_integer_product(None, 64, None, None, 64, None, 0, None, n, dout, 64, F16, None, dout, None),
                L.jarq_integer_linear(None, F16, 64, None, 64, None, 0, None, n, dout, 64, F16, None, dout, None, 0, None)}

    for n, dout in ((0, MOST + 1), (0, 2 ** 31 - 1), (MOST + 1, 8), (2 ** 31 - 1, 8)):
        assert layer(n, dout) == {jarq.JARQ_ERR_ARG}
    assert layer(0, MOST) == {jarq.JARQ_OK}
    assert L.jarq_quantize_rows(None, F16, 0, MOST, MOST, None, MOST, None, None) == jarq.JARQ_OK
