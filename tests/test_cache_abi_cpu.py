"""Refusals of the operators around the paged cache, and what the binding makes of their arguments: host only."""
import ctypes

import pytest

from paper_2602_05305_amd import flashblock as fb

FAKE = 0x1000        # aligned, never dereferenced: validation fails first
ODD = 0x1008


def _shape(**kw):
    base = dict(batch=2, n_q_heads=4, n_kv_heads=2, head_dim=64, block_len=3, prefix_len=128, dtype="bf16")
    base.update(kw)
    return fb.make_shape(**base)


def _rows(**kw):
    base = dict(struct_size=ctypes.sizeof(fb.fb_rows), reserved=0, data=FAKE, batch_stride=3 * 4 * 64, head_stride=64, row_stride=4 * 64)
    base.update(kw)
    return fb.fb_rows(**base)


def _rotary(axis_pairs=(32,), **kw):
    base = dict(struct_size=ctypes.sizeof(fb.fb_rotary), layout=0, n_axes=len(axis_pairs), axis_pairs=(ctypes.c_int32 * 4)(*axis_pairs), offset=0,
                inv_freq=FAKE, positions=None, position_stride=0, first=None)
    base.update(kw)
    return fb.fb_rotary(**base)


def _paged(**kw):
    base = dict(struct_size=ctypes.sizeof(fb.fb_paged_kv), num_pages=8, page_size=64, max_pages=2, k_pool=FAKE, v_pool=FAKE, block_table=FAKE,
                prefix_lens=FAKE)
    base.update(kw)
    return fb.fb_paged_kv(**base)


def _ref(x):
    return None if x is None else ctypes.byref(x)


def _rotate(shape=None, rotary=0, inverse=0, q=0, k=0, v=0, q_out=0, k_out=0, v_out=0):
    views = [_rows() if x == 0 else x for x in (q, k, v, q_out, k_out, v_out)]
    return fb.load_library().fb_rotate_block(_ref(shape or _shape()), _ref(_rotary() if rotary == 0 else rotary), inverse, *map(_ref, views), None)


def test_struct_sizes():
    assert ctypes.sizeof(fb.fb_rotary) == 64 and fb.fb_rotary.inv_freq.offset == 32
    assert ctypes.sizeof(fb.fb_rows) == 40 and fb.fb_rows.batch_stride.offset == 16


@pytest.mark.parametrize("kw,status", [
    (dict(rotary=None), fb.FB_ERR_NULL),
    (dict(q=None), fb.FB_ERR_NULL), (dict(k_out=None), fb.FB_ERR_NULL), (dict(v=None), fb.FB_ERR_NULL),
    (dict(q=None, k=None, v=None, q_out=None, k_out=None, v_out=None), fb.FB_ERR_NULL),
    (dict(inverse=2), fb.FB_ERR_SHAPE), (dict(inverse=-1), fb.FB_ERR_SHAPE),
    (dict(rotary=_rotary(struct_size=8)), fb.FB_ERR_SHAPE), (dict(rotary=_rotary(layout=2)), fb.FB_ERR_SHAPE),
    (dict(rotary=_rotary(n_axes=0)), fb.FB_ERR_SHAPE), (dict(rotary=_rotary(n_axes=5)), fb.FB_ERR_SHAPE),
    (dict(rotary=_rotary((33,))), fb.FB_ERR_SHAPE), (dict(rotary=_rotary((0,))), fb.FB_ERR_SHAPE), (dict(rotary=_rotary((34, -2), positions=FAKE)), fb.FB_ERR_SHAPE),
    (dict(rotary=_rotary(((1 << 31) - 1,))), fb.FB_ERR_SHAPE),
    (dict(rotary=_rotary((16, 16))), fb.FB_ERR_NULL),                       # two axes without positions
    (dict(rotary=_rotary(inv_freq=None)), fb.FB_ERR_NULL), (dict(rotary=_rotary(inv_freq=ODD)), fb.FB_ERR_ALIGN),
    (dict(rotary=_rotary(positions=FAKE + 2)), fb.FB_ERR_ALIGN), (dict(rotary=_rotary(first=FAKE + 1)), fb.FB_ERR_ALIGN),
    (dict(rotary=_rotary(positions=FAKE, position_stride=-1)), fb.FB_ERR_SHAPE), (dict(rotary=_rotary(positions=FAKE, offset=1)), fb.FB_ERR_SHAPE),
    (dict(q=_rows(struct_size=1)), fb.FB_ERR_SHAPE), (dict(q=_rows(reserved=1)), fb.FB_ERR_SHAPE), (dict(v=_rows(data=None)), fb.FB_ERR_NULL),
    (dict(k=_rows(data=ODD)), fb.FB_ERR_ALIGN), (dict(k_out=_rows(data=ODD)), fb.FB_ERR_ALIGN),
    (dict(q=_rows(row_stride=4)), fb.FB_ERR_ALIGN), (dict(q=_rows(head_stride=-64)), fb.FB_ERR_SHAPE),
    (dict(q=_rows(batch_stride=1 << 62)), fb.FB_ERR_SHAPE),
    (dict(q_out=_rows(row_stride=0)), fb.FB_ERR_SHAPE), (dict(k_out=_rows(head_stride=32)), fb.FB_ERR_SHAPE),
    (dict(shape=_shape(head_dim=96)), fb.FB_ERR_UNSUPPORTED), (dict(shape=_shape(dtype=5)), fb.FB_ERR_DTYPE), (dict(shape=_shape(block_len=0)), fb.FB_ERR_SHAPE),
])
def test_rotate_refusals(kw, status):
    assert _rotate(**kw) == status


def _append(shape=None, kv=0, rotary=0, k=0, v=0, counts=None, q=None, q_out=None, lens_out=None):
    return fb.load_library().fb_append_paged(_ref(shape or _shape()), _ref(_paged() if kv == 0 else kv), _ref(_rotary() if rotary == 0 else rotary),
                                             _ref(_rows() if k == 0 else k), _ref(_rows() if v == 0 else v), counts, _ref(q), _ref(q_out), lens_out, None)


@pytest.mark.parametrize("kw,status", [
    (dict(kv=None), fb.FB_ERR_NULL), (dict(k=None), fb.FB_ERR_NULL), (dict(v=None), fb.FB_ERR_NULL), (dict(q=_rows()), fb.FB_ERR_NULL),
    (dict(q_out=_rows()), fb.FB_ERR_NULL), (dict(rotary=None, q=_rows(), q_out=_rows()), fb.FB_ERR_NULL),
    (dict(kv=_paged(struct_size=3)), fb.FB_ERR_SHAPE), (dict(kv=_paged(k_pool=None)), fb.FB_ERR_NULL), (dict(kv=_paged(v_pool=None)), fb.FB_ERR_NULL),
    (dict(kv=_paged(block_table=None)), fb.FB_ERR_NULL), (dict(kv=_paged(prefix_lens=None)), fb.FB_ERR_NULL),
    (dict(kv=_paged(num_pages=0)), fb.FB_ERR_SHAPE), (dict(kv=_paged(page_size=0)), fb.FB_ERR_SHAPE), (dict(kv=_paged(max_pages=1)), fb.FB_ERR_SHAPE),
    (dict(kv=_paged(k_pool=ODD)), fb.FB_ERR_ALIGN), (dict(kv=_paged(v_pool=ODD)), fb.FB_ERR_ALIGN),
    (dict(kv=_paged(block_table=FAKE + 2)), fb.FB_ERR_ALIGN), (dict(counts=FAKE + 1), fb.FB_ERR_ALIGN), (dict(lens_out=0x2002), fb.FB_ERR_ALIGN),
    (dict(lens_out=FAKE), fb.FB_ERR_UNSUPPORTED), (dict(lens_out=FAKE + 4), fb.FB_ERR_UNSUPPORTED), (dict(lens_out=FAKE - 4), fb.FB_ERR_UNSUPPORTED),
    (dict(rotary=_rotary(layout=9)), fb.FB_ERR_SHAPE), (dict(k=_rows(data=ODD)), fb.FB_ERR_ALIGN), (dict(v=_rows(row_stride=1)), fb.FB_ERR_ALIGN),
    (dict(q=_rows(), q_out=_rows(row_stride=0)), fb.FB_ERR_SHAPE), (dict(shape=_shape(prefix_len=-1)), fb.FB_ERR_SHAPE),
])
def test_append_refusals(kw, status):
    assert _append(**kw) == status


class Tensor:
    """What the binding asks of a tensor."""

    def __init__(self, at=4096, strides=(768, 64, 256, 1)):
        self.at, self.strides = at, strides

    def data_ptr(self):
        return self.at

    def stride(self, i=None):
        return self.strides if i is None else self.strides[i]

    def dim(self):
        return len(self.strides)


def test_native_and_python_marshalling_agree():
    """Both forms hand over the same rows, structures and handles."""
    if fb._fbcall is None:
        pytest.skip("fb_call.c is not built")
    seen = []

    def take(*a):
        seen.append(a)
        return 0
    shape, kv, rot = _shape(), _paged(), _rotary()
    q, k, v, o, ko, vo = (Tensor(4096 * (i + 1), (768 + 64 * i, 64, 256, 1)) for i in range(6))
    calls = {
        "fb_rotate_block": [(shape, rot, q, k, v, o, ko, vo, 1, 77), (shape, rot, None, k, None, None, ko, None, 0, 77), (shape, rot, q, None, None, o, None, None, 0, 0)],
        "fb_append_paged": [(shape, kv, rot, k, v, o, q, ko, vo, 5), (shape, kv, None, k, v, None, None, None, None, 5)],
    }
    for name, args_of in calls.items():
        kinds = fb._CACHE_KINDS[name]
        fn = getattr(fb, name).__wrapped__
        names = fn.__code__.co_varnames[:fn.__code__.co_argcount]
        kinds, order = kinds if isinstance(kinds, tuple) else (kinds, " ".join(names))
        callback = ctypes.CFUNCTYPE(ctypes.c_int, *[ctypes.c_int64] * 20)(lambda *a: take(*[
            bytes((ctypes.c_char * 40).from_address(x)) if kind == "R" and x else x for kind, x in zip(kinds + " " * 20, a)]))
        native = fb._fbcall.Call(name, names, fn.__defaults__ or (), kinds, tuple(names.index(x) for x in order.split()),
                                 lambda _: ctypes.cast(callback, ctypes.c_void_p).value, lambda: 0, fb._check, fb.fb_shape, fb.fb_paged_kv, fb.fb_rotary)
        for args in args_of:
            native(*args)
            want = []

            class Lib:
                def __getattr__(self, _):
                    return lambda *a: want.append([bytes(x._obj) if isinstance(getattr(x, "_obj", None), fb.fb_rows) else
                                                   ctypes.addressof(x._obj) if hasattr(x, "_obj") else x or 0 for x in a]) or 0
            real, fb._lib = fb._lib, Lib()
            try:
                fn(*args)
            finally:
                fb._lib = real
            assert list(seen[-1][:len(want[0])]) == want[0] and not any(seen[-1][len(want[0]):]), (name, args)


def test_views_that_are_none_are_refused():
    bad = _shape(n_kv_heads=3)
    for t in (Tensor(strides=(64, 64, 1)), Tensor(strides=(768, 64, 256, 2))):
        with pytest.raises(ValueError):
            fb.fb_rotate_block(bad, _rotary(), t, None, None, Tensor(), None, None, stream=0)
        with pytest.raises(ValueError):
            fb.make_rows(t)
    with pytest.raises(fb.FlashBlockError):
        fb.fb_rotate_block(bad, _rotary(), Tensor(), None, None, Tensor(), None, None, stream=0)
    with pytest.raises(ValueError):
        fb.make_rotary(Tensor(), [])


def _shared(shape=None, q=FAKE, kv=0, pages=FAKE, shared_len=1000, o=FAKE, m=FAKE, lse=FAKE, ws=FAKE, nbytes=1 << 40, step=None):
    lib, shape = fb.load_library(), shape or _shape()
    kv = _paged() if kv == 0 else kv
    if step is None:
        return lib.fb_external_partial_shared(_ref(shape), q, _ref(kv), pages, shared_len, o, m, lse, ws, nbytes, None)
    kb, vb, out, lse_out = step
    return lib.fb_refresh_step_shared(_ref(shape), q, _ref(kv), pages, shared_len, kb, vb, o, m, lse, out, lse_out, ws, nbytes, None)


@pytest.mark.parametrize("kw,status", [
    (dict(q=None), fb.FB_ERR_NULL), (dict(kv=None), fb.FB_ERR_NULL), (dict(o=None), fb.FB_ERR_NULL), (dict(m=None), fb.FB_ERR_NULL), (dict(lse=None), fb.FB_ERR_NULL),
    (dict(pages=None), fb.FB_ERR_NULL), (dict(kv=_paged(block_table=None)), fb.FB_ERR_NULL), (dict(kv=_paged(prefix_lens=None)), fb.FB_ERR_NULL),
    (dict(kv=_paged(k_pool=None)), fb.FB_ERR_NULL), (dict(kv=_paged(v_pool=None)), fb.FB_ERR_NULL),
    (dict(shared_len=-1), fb.FB_ERR_SHAPE), (dict(shared_len=(1 << 30) + 1), fb.FB_ERR_UNSUPPORTED), (dict(kv=_paged(struct_size=1)), fb.FB_ERR_SHAPE),
    (dict(kv=_paged(num_pages=0)), fb.FB_ERR_SHAPE), (dict(kv=_paged(page_size=0)), fb.FB_ERR_SHAPE), (dict(kv=_paged(max_pages=0)), fb.FB_ERR_SHAPE),
    (dict(kv=_paged(page_size=96)), fb.FB_ERR_UNSUPPORTED), (dict(kv=_paged(max_pages=1)), fb.FB_ERR_SHAPE),
    (dict(q=ODD), fb.FB_ERR_ALIGN), (dict(o=ODD), fb.FB_ERR_ALIGN), (dict(ws=ODD), fb.FB_ERR_ALIGN), (dict(kv=_paged(v_pool=ODD)), fb.FB_ERR_ALIGN),
    (dict(pages=FAKE + 2), fb.FB_ERR_ALIGN), (dict(ws=None), fb.FB_ERR_WORKSPACE), (dict(nbytes=64), fb.FB_ERR_WORKSPACE),
    (dict(shape=_shape(head_dim=32)), fb.FB_ERR_UNSUPPORTED), (dict(shape=_shape(dtype=9)), fb.FB_ERR_DTYPE), (dict(shape=_shape(n_q_heads=3)), fb.FB_ERR_SHAPE),
    (dict(shape=_shape(batch=2, n_q_heads=1 << 14, n_kv_heads=1 << 14, head_dim=128, block_len=1 << 13, prefix_len=0)), fb.FB_ERR_UNSUPPORTED),     # rows further than 32 bits apart
])
def test_shared_refusals(kw, status):
    assert _shared(**kw) == status
    assert _shared(**kw, step=(FAKE, FAKE, FAKE, None)) == status


def test_shared_step_refusals():
    for step, status in (((None, FAKE, FAKE, FAKE), fb.FB_ERR_NULL), ((FAKE, None, FAKE, FAKE), fb.FB_ERR_NULL), ((FAKE, FAKE, None, FAKE), fb.FB_ERR_NULL),
                         ((ODD, FAKE, FAKE, FAKE), fb.FB_ERR_ALIGN), ((FAKE, FAKE, ODD, FAKE), fb.FB_ERR_ALIGN), ((FAKE, FAKE, FAKE, ODD), fb.FB_ERR_ALIGN)):
        assert _shared(step=step) == status


def test_shared_workspace_query():
    s = _shape()
    assert fb.fb_shared_workspace_bytes(s, 0) >= 256
    assert fb.fb_shared_workspace_bytes(s, 1 << 20) > fb.fb_shared_workspace_bytes(s, 64)
    assert fb.fb_shared_workspace_bytes(_shape(prefix_len=0), 0) >= 256
    assert fb.fb_shared_workspace_bytes(s, -1) == 0 and fb.fb_shared_workspace_bytes(_shape(batch=0), 64) == 0 and fb.fb_shared_workspace_bytes(s, (1 << 30) + 1) == 0
    n = fb.fb_shared_workspace_bytes(s, 1000)
    assert _shared(nbytes=n - 1) == fb.FB_ERR_WORKSPACE


@pytest.mark.parametrize("kw", [
    dict(counts=0x2000, lens_out=0x2000), dict(counts=0x2000, lens_out=0x2004), dict(counts=0x2004, lens_out=0x2000),
    dict(kv=_paged(block_table=0x2000), lens_out=0x200c), dict(rotary=_rotary(first=0x2000), lens_out=0x2000),
    dict(rotary=_rotary(positions=0x2000), lens_out=0x2008), dict(rotary=_rotary(positions=0x2000, position_stride=100), lens_out=0x2000 + 400 + 8),
])
def test_new_lengths_over_what_other_workgroups_read_are_refused(kw):
    """batch 2, block_len 3, two pages a sequence"""
    assert _append(**kw) == fb.FB_ERR_UNSUPPORTED


def test_shared_counts_keys_in_32_bits():
    long = _shape(prefix_len=(1 << 30) + 1)
    kv = _paged(max_pages=1 << 25)
    assert _shared(shape=long, kv=kv) == fb.FB_ERR_UNSUPPORTED
    assert _shared(shape=long, kv=kv, step=(FAKE, FAKE, FAKE, None)) == fb.FB_ERR_UNSUPPORTED
    assert fb.fb_shared_workspace_bytes(long, 64) == 0
