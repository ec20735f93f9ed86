"""What the binding hands to the entry points of the operators beside the layer, and what it refuses.  No GPU: the tensors are on the host and
say that they are on a device, and a stand-in takes the calls."""
import ctypes as C

import pytest
import torch

from paper_2510_26730_amd import binding as ef


class Device(torch.Tensor):
    """A tensor in host memory that counts as the first device's."""

    def get_device(self):
        return 0


def dev(t):
    return t.as_subclass(Device)


class Calls:
    """Takes the calls of the library; ef_quant_rows* write what the entry points may write."""

    def __init__(self):
        self.made = []

    def __getattr__(self, name):
        def call(*args):
            self.made.append((name, args))
            if name == "ef_quant_rows":
                x, kind, ldx, rows, K, codes, ldc, scales, s = args
                self.zero(codes, rows, K, ldc, ldc)
            elif name == "ef_quant_rows_within":
                x, kind, ldx, rows, K, codes, width, ldc, scales, s = args
                self.zero(codes, rows, K, width, ldc)
            return 1 << 20 if name.endswith("_work") else 0
        return call

    @staticmethod
    def zero(codes, rows, K, width, ldc):
        for r in range(rows):
            C.memset(codes + r * ldc, 0, min((K + 63) // 64 * 64, width))


@pytest.fixture
def calls(monkeypatch):
    c = Calls()
    monkeypatch.setattr(ef, "lib", lambda: c)
    return c


@pytest.mark.parametrize("rows,first,last", [(4, 100, 200), (4, 0, 100), (1, 100, 200), (3, 30, 190), (2, 0, 200)])
def test_codes_in_columns_of_a_wider_matrix(calls, rows, first, last):
    """Nothing behind the columns is written, not in the next row and not behind the last one."""
    room = torch.full((rows * 200 + 256,), 99, dtype=torch.int8)
    codes = dev(room[:rows * 200].view(rows, 200)[:, first:last])
    ef.ef_quant_rows(dev(torch.zeros(rows, 100)), codes, dev(torch.zeros(rows)))
    assert len(calls.made) == 1
    wide = room[:rows * 200].view(rows, 200)
    assert (room[rows * 200:] == 99).all() and (wide[:, :first] == 99).all() and (wide[:, last:] == 99).all()
    assert (wide[:, first:first + 100] == 0).all()


def test_width_is_checked():
    refuse = lambda width, ldc: ef.lib().ef_quant_rows_within(4096, ef.EF_BF16, 64, 2, 64, 4096, width, ldc, 4096, None)  # noqa: E731
    for width, ldc in ((63, 64), (65, 64), (200, 128)):
        assert refuse(width, ldc) == ef.EF_EINVAL and "width" in ef.ef_last_error(None)


def test_tokens_of_a_launch_are_checked():
    for k, most in ((1, (1 << 29) - 64), (4, (1 << 29) - 64), (8, (1 << 28) - 1)):
        assert ef.ef_route_scores_work(most, 16, k) > 0 and ef.ef_route_scores_work(most + 1, 16, k) == 0


class Other(torch.Tensor):
    def get_device(self):
        return 1


def zeros(*shape, t=torch.float32):
    return dev(torch.zeros(*shape, dtype=t))


def i32(*shape):
    return zeros(*shape, t=torch.int32)


def route_args(**kw):
    a = dict(logits=zeros(5, 16), bias=zeros(16), ids=i32(5, 2), w=zeros(5, 2), counts=i32(16), offsets=i32(17), perm=i32(10), inv_perm=i32(10),
             work=zeros(1 << 16, t=torch.uint8))
    a.update(kw)
    return a


def product_args(**kw):
    a = dict(a=zeros(5, 64, t=torch.int8), w=zeros(3, 32, 64, t=torch.int8), w_scale=zeros(3, 32), out=zeros(10, 16), work=zeros(1 << 16, t=torch.uint8),
             a_scale=zeros(5), rows=i32(10), row_div=2, offsets=i32(4), swiglu=True)
    a.update(kw)
    return a


def combine_args(**kw):
    a = dict(y=zeros(10, 24), w=zeros(5, 2), inv_perm=i32(10), out=zeros(5, 24))
    a.update(kw)
    return a


def quant_args(**kw):
    a = dict(x=zeros(5, 32), codes=zeros(5, 64, t=torch.int8), scales=zeros(5))
    a.update(kw)
    return a


CALLS = {"route": (ef.ef_route_scores, route_args), "product": (ef.ef_matmul_q8, product_args), "combine": (ef.ef_combine, combine_args),
         "quant": (ef.ef_quant_rows, quant_args)}
# operands of fixed types: what they hold at least, and whether they may be left out
VECTORS = [("route", "bias", (16,)), ("route", "ids", (5, 2)), ("route", "w", (5, 2)), ("route", "counts", (16,)), ("route", "offsets", (17,)),
           ("route", "perm", (10,)), ("route", "inv_perm", (10,)), ("product", "w_scale", (3, 32)), ("product", "a_scale", (5,)),
           ("product", "rows", (10,)), ("product", "offsets", (4,)), ("combine", "w", (5, 2)), ("combine", "inv_perm", (10,)), ("quant", "scales", (5,))]


@pytest.mark.parametrize("call", CALLS)
def test_operands_that_fit_are_taken(calls, call):
    f, args = CALLS[call]
    f(**args())
    assert len(calls.made) == 1


@pytest.mark.parametrize("call,name,shape", VECTORS, ids=lambda v: v if isinstance(v, str) else "")
def test_operands_of_the_wrong_type_are_refused(calls, call, name, shape):
    """Of 64 or 16 bits, as sorting and gates leave them: they would be read as 32-bit words."""
    f, args = CALLS[call]
    right = args()[name].dtype
    for t in (torch.int64, torch.int16, torch.bfloat16, torch.float64, torch.int32 if right is torch.float32 else torch.float32):
        with pytest.raises(ef.EfError, match=name):
            f(**args(**{name: zeros(*shape, t=t)}))
    assert not calls.made


@pytest.mark.parametrize("call,name,shape", VECTORS, ids=lambda v: v if isinstance(v, str) else "")
def test_operands_that_are_too_small_or_elsewhere_are_refused(calls, call, name, shape):
    f, args = CALLS[call]
    right = args()[name].dtype
    short = (shape[0] - 1,) + shape[1:]
    for x in (zeros(*short, t=right), zeros(*shape, 2, t=right)[..., 0], torch.zeros(shape, dtype=right),
              torch.zeros(shape, dtype=right).as_subclass(Other), torch.zeros(shape).numpy()):
        with pytest.raises(ef.EfError):
            f(**args(**{name: x}))
    assert not calls.made


@pytest.mark.parametrize("call,name", [("route", "logits"), ("route", "work"), ("product", "a"), ("product", "w"), ("product", "out"), ("product", "work"),
                                       ("combine", "y"), ("combine", "out"), ("quant", "x"), ("quant", "codes")])
def test_matrices_and_scratch_elsewhere_are_refused(calls, call, name):
    f, args = CALLS[call]
    x = args()[name]
    for other in (torch.zeros(x.shape, dtype=x.dtype), torch.zeros(x.shape, dtype=x.dtype).as_subclass(Other)):
        with pytest.raises(ef.EfError, match="device|GPU| on "):
            f(**args(**{name: other}))
    assert not calls.made


def test_scratch_that_is_not_consecutive_is_refused(calls):
    for call in ("route", "product"):
        f, args = CALLS[call]
        with pytest.raises(ef.EfError, match="consecutive"):
            f(**args(work=zeros(1 << 16, 2, t=torch.uint8)[:, 0]))
    assert not calls.made


def test_what_may_be_left_out_or_given_as_an_address(calls):
    ef.ef_route_scores(**route_args(bias=None, perm=4096))
    ef.ef_matmul_q8(**product_args(a=zeros(10, 64), a_scale=None, rows=None, work=None))
    ef.ef_combine(**combine_args(inv_perm=None))
    assert [name for name, _ in calls.made] == ["ef_route_scores_of", "ef_matmul_q8", "ef_combine"]


def test_packed_structures(calls):
    """The bytes that the binding makes are the header's structures."""
    class Operands(C.Structure):
        _fields_ = [(n, C.c_void_p) for n in ("logits", "bias", "topk_ids", "topk_w", "counts", "offsets", "perm", "inv_perm", "work")] + [
            ("work_bytes", C.c_size_t), ("ld", C.c_int64), ("type", C.c_int32), ("T", C.c_int32)]
    a = route_args(logits=zeros(5, 20)[:, :16])
    ef.ef_route_scores(**a, sigmoid=True, n_groups=4, groups_kept=2, group_best=2, renorm=True, scale=2.5)
    r, o = calls.made[-1][1][:2]
    r, o = ef.ef_router.from_buffer_copy(r), Operands.from_buffer_copy(o)
    assert (r.n_experts, r.top_k, r.score, r.n_groups, r.groups_kept, r.group_best, r.renorm, r.scale) == (16, 2, 1, 4, 2, 2, 1, 2.5)
    for field, name in (("logits", "logits"), ("bias", "bias"), ("topk_ids", "ids"), ("topk_w", "w"), ("counts", "counts"), ("offsets", "offsets"),
                        ("perm", "perm"), ("inv_perm", "inv_perm"), ("work", "work")):
        assert getattr(o, field) == a[name].data_ptr()
    assert (o.work_bytes, o.ld, o.type, o.T) == (1 << 16, 20, ef.EF_F32, 5)
    a = product_args()
    ef.ef_matmul_q8(**a)
    assert len(calls.made[-1][1][0]) == C.sizeof(ef.ef_q8_product)
    p = ef.ef_q8_product.from_buffer_copy(calls.made[-1][1][0])
    for name in ("a", "a_scale", "rows", "offsets", "w", "w_scale", "out"):
        assert getattr(p, name) == a[name].data_ptr()
    assert (p.lda, p.ldw, p.w_group, p.ldo, p.a_type, p.out_type, p.a_rows, p.M, p.N, p.K, p.G, p.row_div, p.swiglu) == (
        64, 64, 2048, 16, ef.EF_I8, ef.EF_F32, 5, 10, 32, 64, 3, 2, 1)


def test_operands_in_a_structure_are_checked():
    assert ef.lib().ef_route_scores_of(bytes(ef.ef_router(8, 2, 0, 1, 1, 1, 0, 1.0)), None, None) == ef.EF_EINVAL
    assert ef.lib().ef_route_scores_of(bytes(ef.ef_router(8, 9, 0, 1, 1, 1, 0, 1.0)), bytes(96), None) == ef.EF_EINVAL
    assert "top_k" in ef.ef_last_error(None)


# ---- the layer of the operators ------------------------------------------------------------------

@pytest.fixture
def layer(calls, monkeypatch):
    """A Q8Layer of 4 experts, d = 64, F = 32, for 6 tokens, whose tensors count as a device's."""
    from paper_2510_26730_amd.q8_layer import Q8Layer
    monkeypatch.setattr(torch.Tensor, "get_device", lambda self: 0)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: 4096)
    made = Q8Layer(torch.zeros(4, 64, 64), torch.zeros(4, 64, 32), 2, 6)
    calls.made.clear()
    return made


def test_layer_takes_inputs_that_fit(layer, calls):
    for T in (0, 1, 6):
        out = layer(torch.zeros(T, 64), torch.zeros(T, 4))
        assert out.shape == (T, 64) and layer.ids.shape == (T, 2)
    assert [n for n, _ in calls.made] == ["ef_route_scores_of", "ef_matmul_q8", "ef_matmul_q8", "ef_combine"] * 3


@pytest.mark.parametrize("hidden,logits,out", [
    ((3, 64), (4, 4), None), ((3, 64), (6, 4), None), ((3, 64), (9, 4), None), ((3, 64), (2, 4), None), ((3, 64), (3, 5), None),
    ((3, 64), (3, 3), None), ((3, 64), (3, 400), None), ((3, 64), (12,), None), ((3, 32), (3, 4), None), ((3, 128), (3, 4), None), ((7, 64), (7, 4), None),
    ((3, 64), (3, 4), (4, 64)), ((3, 64), (3, 4), (2, 64)), ((3, 64), (3, 4), (3, 32)), ((192,), (3, 4), None)])
def test_layer_refuses_inputs_that_do_not_fit(layer, calls, hidden, logits, out):
    """Before its first call: routing more tokens than there are would write behind the buffers' views."""
    with pytest.raises(ef.EfError):
        layer(torch.zeros(*hidden), torch.zeros(*logits), None if out is None else torch.zeros(*out))
    assert not calls.made


@pytest.mark.parametrize("stream", [8192, "object"])
def test_layer_allocates_where_it_writes(layer, calls, monkeypatch, stream):
    """The memory of an output belongs to the stream that writes it: allocated on another, it may still be in use there, and be given out again
    too early."""
    entered = []

    class On:
        def __init__(self, s):
            self.s = s

        def __enter__(self):
            entered.append(self.s)

        def __exit__(self, *a):
            entered.pop()

    class Stream:
        def __init__(self, handle, device=None):
            self.cuda_stream = handle

    where = []
    empty = torch.empty
    monkeypatch.setattr(torch.cuda, "stream", On)
    monkeypatch.setattr(torch.cuda, "ExternalStream", Stream)
    monkeypatch.setattr(torch, "empty", lambda *a, **kw: (where.extend(s.cuda_stream for s in entered), empty(*a, **kw))[1])
    x, z = torch.zeros(3, 64), torch.zeros(3, 4)
    layer(x, z, stream=stream if stream == 8192 else Stream(8192))
    assert where == [8192]
    assert all(args[-1] == 8192 for _, args in calls.made)
    layer(x, z)
    layer(x, z, torch.zeros(3, 64), stream=8192)
    assert where == [8192] and not entered
