"""The workspace of santa_attend_chunk and santa_decode_window on the host (no GPU): it follows the
tokens to expect, not the rows of a padded batch, and refusals by size follow the launch."""

import ctypes

import pytest

from paper_2605_01910_amd import santa as S

ref = ctypes.byref


def size(B=1, n_k=32768, tokens=1, most=1, Hq=32, Hkv=8, dtype=0, window=None):
    kv = S.santa_kv_t(16, 16, n_k * Hkv * 128, Hkv * 128, 128, None, None, 0, 0, n_k)
    sh, ch = S.santa_shape_t(B, Hq, Hkv, 128, dtype), S.santa_chunk_t(16, tokens, most)
    win = None if window is None else ref(S.window_of(*window))
    return S.load().santa_attend_workspace_size(ref(sh), ref(kv), ref(ch), win)


@pytest.mark.parametrize("B,most,rows,n_k", [(1, 1, 2001, 32768), (4, 1, 8196, 131072), (1, 8, 4096, 65536),
                                             (3, 40, 20000, 32768), (16, 5, 2 ** 20, 65536)])
@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("G", [1, 4, 8])
def test_padding_needs_no_room(B, most, rows, n_k, dtype, G):
    """Rows that no sequence holds: the workspace is the unpadded batch's."""
    for window in (None, (4096, 4)):
        kw = dict(B=B, n_k=n_k, most=most, Hq=8 * G, Hkv=8, dtype=dtype, window=window)
        assert 0 < size(tokens=rows, **kw) == size(tokens=B * most, **kw)


@pytest.mark.parametrize("most", [0, 1, 8, 100, 5000])
@pytest.mark.parametrize("rows", [1, 300, 8192, 2 ** 20, 2 ** 25])
@pytest.mark.parametrize("B", [1, 16, 4096])
def test_partial_results_are_bounded(B, rows, most):
    """At most 512 workgroups are split (two for each of 256 CUs), 128 rows of 520 bytes each, beside
    the head that every call's workspace has; one split of each KV head's tile may pass that."""
    head = size(n_k=1)
    for n_k in (100, 32768, 2 ** 20):
        for Hkv in (1, 8, 64):
            assert 0 < size(B, n_k, rows, most, Hkv, Hkv) - head <= 512 * 128 * 520 + 512 or \
                size(B, n_k, rows, most, Hkv, Hkv) == head


@pytest.mark.parametrize("Hq,Hkv,most", [(128, 128, 1), (128, 128, 0), (64, 8, 0), (8, 1, 0), (64, 8, 2 ** 20)])
def test_long_batches_are_not_refused(Hq, Hkv, most):
    """2^25 rows, the most that a call may have.  (A missing workspace is refused after the launch's
    size is, so no launch is made here.)"""
    kv = S.santa_kv_t(16, 16, 0, Hkv * 128, 128, None, None, 0, 0, 4096)
    sh, ch = S.santa_shape_t(1, Hq, Hkv, 128, 0), S.santa_chunk_t(16, 2 ** 25, most)
    assert S.load().santa_attend_chunk(16, ref(kv), ref(sh), ref(ch), None, 0.1, 16, None, 0, None) == S.SANTA_ERR_WORKSPACE


def test_launches_that_do_not_fit_are_refused():
    kv = S.santa_kv_t(16, 16, 0, 0, 128, None, None, 0, 0, 4096)
    sh = S.santa_shape_t(1, 2 ** 24 + 8, 2 ** 24 + 8, 128, 0)
    assert S.load().santa_attend_chunk(16, ref(kv), ref(sh), None, None, 0.1, 16, None, 0, None) == S.SANTA_ERR_UNSUPPORTED
    sh, ch = S.santa_shape_t(4096, 32, 32, 128, 0), S.santa_chunk_t(16, 2 ** 21, 0)
    with S.options("auto", 256):
        assert S.load().santa_attend_chunk(16, ref(kv), ref(sh), ref(ch), None, 0.1, 16, None, 0, None) == S.SANTA_ERR_UNSUPPORTED


def test_no_size_for_calls_that_are_refused():
    assert size() > 0 and size(dtype=1) > 0
    kv = S.santa_kv_t(16, 16, 0, 128, 128, None, None, 0, 0, 4096)
    for dtype, kv_dtype, fine in ((0, 0, True), (0, 1, True), (1, 0, True), (1, 1, False), (0, 2, False), (0, -1, False)):
        kv.kv_dtype = kv_dtype
        sh = S.santa_shape_t(2, 8, 2, 128, dtype)
        assert (S.load().santa_attend_workspace_size(ref(sh), ref(kv), None, None) > 0) == fine
    assert size(Hq=2 ** 24 + 8, Hkv=2 ** 24 + 8, n_k=1) == 0


def test_more_keys_than_32_bits_number_are_refused():
    """A contiguous cache whose rows share memory (stride 0) or a table that names one page throughout
    can have as many keys as n_k says."""
    sh, ch = S.santa_shape_t(2, 8, 2, 128, 0), S.santa_chunk_t(16, 10, 5)
    for n_k, fine in ((2 ** 30, True), (2 ** 30 + 1, False), (2 ** 31 - 1, False)):
        kv = S.santa_kv_t(16, 16, 0, 0, 128, None, None, 0, 0, n_k)
        status = S.SANTA_ERR_WORKSPACE if fine else S.SANTA_ERR_UNSUPPORTED
        assert S.load().santa_attend_chunk(16, ref(kv), ref(sh), ref(ch), None, 0.1, 16, None, 0, None) == status
        assert (S.load().santa_attend_workspace_size(ref(sh), ref(kv), ref(ch), None) > 0) == fine
