"""Host-side checks of the operators behind the feature maps (no GPU): arguments that must be refused before anything is enqueued."""
import ctypes as C

import pytest

from paper_2210_09887_amd import binding as B

FAKE = 0x7F0000000000          # an aligned address that is never dereferenced on the host


def refused(status, call, *args):
    with pytest.raises(B.MdcnnError) as e:
        call(*args)
    assert e.value.status == status and B.mdcnn_last_error()


def norm_desc(**kw):
    N, H, W, Cc = kw.get("N", 2), kw.get("H", 6), kw.get("W", 5), kw.get("C", 16)
    s = B.mdcnn_strides(H * W * Cc, W * Cc, Cc)
    d = B.mdcnn_group_norm_desc(N, H, W, Cc, 4, B.MDCNN_F16, B.MDCNN_ACT_SILU, 1e-5, None, None, s, s, s)
    for k, v in kw.items():
        setattr(d, k, v)
    return d


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=3), 3), (dict(dtype=-1), 3), (dict(N=-1), 2), (dict(H=0), 2), (dict(W=0), 2), (dict(groups=0), 2), (dict(groups=3), 2), (dict(C=4100), 5),
    (dict(H=1 << 13, W=1 << 12), 5), (dict(act=3), 2), (dict(eps=-1.0), 2), (dict(eps=float("nan")), 2), (dict(xs=B.mdcnn_strides(-1, 80, 16)), 2),
    (dict(ys=B.mdcnn_strides(480, 80, 15)), 2), (dict(ys=B.mdcnn_strides(480, 79, 16)), 2), (dict(ys=B.mdcnn_strides(479, 80, 16)), 2), (dict(gamma_dev=FAKE + 2), 4)])
def test_group_norm_descriptors(kw, status):
    refused(status, B.mdcnn_group_norm_bytes, norm_desc(**kw))
    refused(status, B.mdcnn_group_norm, norm_desc(**kw), FAKE, FAKE, FAKE, FAKE, FAKE, 1 << 30)


def test_group_norm_arguments():
    big = dict(H=300, W=300)                             # does not fit the registers of a block: needs a workspace
    n = B.mdcnn_group_norm_bytes(norm_desc(**big))
    assert n > 0 and B.mdcnn_group_norm_bytes(norm_desc()) == 0
    call = B.mdcnn_group_norm
    refused(5, call, norm_desc(**big), FAKE, FAKE, FAKE, FAKE, FAKE, n - 1)
    refused(1, call, norm_desc(**big), FAKE, FAKE, FAKE, FAKE, None, n)
    refused(4, call, norm_desc(**big), FAKE, FAKE, FAKE, FAKE, FAKE + 8, n)
    refused(4, call, norm_desc(**big), FAKE + 1, FAKE, FAKE, FAKE, FAKE, n)
    for k in range(4):
        args = [FAKE] * 4
        args[k] = None
        refused(1, call, norm_desc(**big), *args, FAKE, n)
    n = B.mdcnn_group_norm_bytes(norm_desc(**big), True)
    call = B.mdcnn_group_norm_backward
    refused(5, call, norm_desc(**big), *[FAKE] * 8, n - 1)
    refused(2, call, norm_desc(ds=B.mdcnn_strides(0, 0, -1), **big), *[FAKE] * 8, n)
    for k in range(7):
        args = [FAKE] * 7
        args[k] = None
        refused(1, call, norm_desc(**big), *args, FAKE, n)
    assert B.lib().mdcnn_group_norm_bytes(None, 0, C.byref(C.c_size_t())) == 1
    assert B.lib().mdcnn_group_norm_bytes(C.byref(norm_desc()), 0, None) == 1


def rotary_desc(**kw):
    d = B.mdcnn_rotary_desc(32, 2, 10000.0, B.MDCNN_ROTARY_PARTS, 4.0, 4096.0, 1.0, 32.0)
    for k, v in kw.items():
        setattr(d, k, v)
    return d


@pytest.mark.parametrize("kw", [dict(turned=0), dict(turned=30), dict(turned=33), dict(axes=0), dict(axes=5), dict(base=1.0), dict(base=float("nan")), dict(base=float("inf")),
                                dict(scaling=4), dict(factor=0.5), dict(factor=float("inf")), dict(original=0.0), dict(slow=-1.0), dict(fast=1.0)])
def test_rotary_tables(kw):
    refused(2, B.mdcnn_rotary_table, rotary_desc(**kw))


def test_rotary_table_values():
    import math
    steps = B.mdcnn_rotary_table(rotary_desc(scaling=B.MDCNN_ROTARY_PLAIN))
    assert len(steps) == 16 and steps[:8] == steps[8:]
    for i, s in enumerate(steps[:8]):
        assert abs(s / 2.0 ** 64 * 2 * math.pi / 10000.0 ** (-i / 8) - 1) < 1e-14
    slow = B.mdcnn_rotary_table(rotary_desc(scaling=B.MDCNN_ROTARY_BASE))
    assert slow[0] == steps[0] and abs(steps[7] / slow[7] - 4) < 1e-12
    assert B.mdcnn_rotary_table(rotary_desc(scaling=B.MDCNN_ROTARY_BASE, turned=2, axes=1)) == steps[:1]


def heads(**kw):
    m = B.mdcnn_heads(FAKE, FAKE, 4, 128, 32, 128, 32)
    for k, v in kw.items():
        setattr(m, k, v)
    return m


@pytest.mark.parametrize("change,status", [
    (dict(dtype=5), 3), (dict(tokens=-1), 2), (dict(dim=1), 5), (dict(dim=257), 5), (dict(turned=34), 2), (dict(turned=0), 2), (dict(turned=30, axes=2), 2), (dict(axes=0), 2),
    (dict(axes=5), 2), (dict(interleaved=2), 2), (dict(inverse=-1), 2), (dict(magnitude=float("nan")), 2), (dict(pos_ptr=None), 1), (dict(steps_ptr=None), 1),
    (dict(pos_ptr=FAKE + 2), 4), (dict(steps_ptr=FAKE + 4), 4), (dict(maps=[]), 2), (dict(maps=[heads()] * 3), 2), (dict(maps=[heads(heads=0)]), 2), (dict(maps=[heads(x_dev=None)]), 1),
    (dict(maps=[heads(y_dev=None)]), 1), (dict(maps=[heads(x_dev=FAKE + 1)]), 4), (dict(maps=[heads(x_token=-1)]), 2), (dict(maps=[heads(y_token=127)]), 2),
    (dict(maps=[heads(y_head=31)]), 2), (dict(maps=[heads(y_token=32, y_head=95)]), 2), (dict(maps=[heads(), heads(y_token=31)]), 2)])
def test_rotary_arguments(change, status):
    kw = dict(maps=[heads()], tokens=3, dim=32, dtype=0, pos_ptr=FAKE, axes=1, steps_ptr=FAKE, turned=32)
    kw.update(change)
    refused(status, lambda: B.mdcnn_rotary(**kw))


def cache(**kw):
    c = B.mdcnn_cache_desc(10, 4, 32, FAKE, FAKE, FAKE, FAKE, FAKE, 3, 5)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def test_cache_pitch():
    assert [B.mdcnn_cache_pitch(d) for d in (0, 4, 7, 8, 12, 32, 40, 64, 72, 96, 104, 128, 136, 192, 200, 256, 264)] == \
        [0, 0, 0, 32, 0, 32, 64, 64, 96, 96, 128, 128, 192, 192, 256, 256, 0]


@pytest.mark.parametrize("call", [B.mdcnn_cache_store, B.mdcnn_cache_read], ids=["store", "read"])
@pytest.mark.parametrize("change,status", [
    (dict(c=dict(dim=30)), 2), (dict(c=dict(heads=0)), 2), (dict(c=dict(pages=-1)), 5), (dict(c=dict(n_seq=-1)), 5), (dict(c=dict(max_pages=-1)), 5), (dict(c=dict(k_dev=None)), 1),
    (dict(c=dict(v_scale_dev=None)), 1), (dict(c=dict(table_dev=None)), 1), (dict(c=dict(v_dev=FAKE + 8)), 4), (dict(c=dict(table_dev=FAKE + 2)), 4), (dict(dtype=3), 3),
    (dict(max_new=-1), 2), (dict(tokens=-1), 2), (dict(starts=None), 1), (dict(at=None), 1), (dict(starts=FAKE + 1), 4), (dict(at=FAKE + 2), 4), (dict(k=dict(heads=3)), 2),
    (dict(v=dict(x_dev=None, y_dev=None)), 1), (dict(k=dict(x_dev=FAKE + 1, y_dev=FAKE + 1)), 4), (dict(c=dict(n_seq=1 << 20), max_new=1 << 30, tokens=1 << 30), 5)])
def test_cache_arguments(call, change, status):
    kw = dict(dtype=1, max_new=100, tokens=200, starts=FAKE, at=FAKE)
    kw.update({k: v for k, v in change.items() if k not in ("c", "k", "v")})
    refused(status, call, cache(**change.get("c", {})), heads(**change.get("k", {})), heads(**change.get("v", {})), kw["tokens"], kw["starts"], kw["at"], kw["max_new"], kw["dtype"])


def attending(**kw):
    a = B.mdcnn_attend_desc(FAKE, FAKE, 6, 2, 300, 0.125, 1, 0, None, 0)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


@pytest.mark.parametrize("change,status", [
    (dict(c=dict(dim=12)), 2), (dict(c=dict(k_dev=None)), 1), (dict(a=dict(tokens=-1)), 2), (dict(a=dict(max_new=-1)), 2), (dict(a=dict(max_len=-1)), 2), (dict(a=dict(causal=2)), 2),
    (dict(a=dict(window=-1)), 2), (dict(a=dict(window=3, causal=0)), 2), (dict(a=dict(scale=float("inf"))), 2), (dict(a=dict(starts_dev=None)), 1),
    (dict(a=dict(lengths_dev=FAKE + 2)), 4), (dict(a=dict(mask_dev=FAKE, mask_row=299)), 5), (dict(q=dict(heads=6)), 2), (dict(q=dict(heads=0)), 2), (dict(q=dict(x_dev=None)), 1),
    (dict(q=dict(y_dev=None)), 1), (dict(q=dict(y_dev=FAKE + 1)), 4), (dict(q=dict(y_token=100)), 2), (dict(dtype=9), 3), (dict(lse=FAKE + 2), 4), (dict(work=FAKE + 8), 4), (dict(n=0), 5),
    (dict(work=None), 1), (dict(c=dict(n_seq=1 << 20), a=dict(tokens=1 << 30, max_new=1 << 30)), 5)])
def test_attend_arguments(change, status):
    big = dict(max_len=100000)
    big.update(change.get("a", {}))
    c, a, q = cache(max_pages=2000, **change.get("c", {})), attending(**big), heads(heads=8, x_token=256, y_token=256)
    for k, v in change.get("q", {}).items():
        setattr(q, k, v)
    refused(status, B.mdcnn_cache_attend, c, a, q, change.get("dtype", 1), change.get("lse", FAKE), change.get("work", FAKE), change.get("n", 1 << 40))


def test_attend_workspace():
    c, a = cache(max_pages=2000), attending(max_len=100000)
    assert B.mdcnn_cache_attend_bytes(c, a, 8, 1) > 0 and B.mdcnn_cache_attend_bytes(c, attending(max_len=100), 8, 1) == 0
    refused(2, B.mdcnn_cache_attend_bytes, c, a, 6, 1)
    refused(3, B.mdcnn_cache_attend_bytes, c, a, 8, 7)


def test_one_token_has_no_token_stride():
    """[heads, 1, dim] seen as [1, heads, dim]: the checks get past the heads to what is refused behind them."""
    for token in (32, 0, 1, 31, 95, 1 << 40):
        one = heads(x_token=max(0, token), y_token=token)
        refused(1, B.mdcnn_rotary, [one], 1, 32, 0, None, 1, FAKE, 32)
        refused(4, B.mdcnn_cache_attend, cache(), attending(tokens=1, max_new=1), one, 1, FAKE + 2, FAKE, 1 << 40)
        refused(4, B.mdcnn_cache_read, cache(), one, heads(y_dev=FAKE + 1), 1, FAKE, FAKE, 1, 1)
    refused(2, B.mdcnn_rotary, [heads(y_head=31)], 1, 32, 0, None, 1, FAKE, 32)          # heads that overlap still do
    refused(2, B.mdcnn_rotary, [heads(y_token=32)], 2, 32, 0, None, 1, FAKE, 32)         # and so do tokens, where there are two


@pytest.mark.parametrize("kw", [dict(max_pages=0, table_dev=None), dict(pages=0, k_dev=None, v_dev=None, k_scale_dev=None, v_scale_dev=None), dict(pages=0, max_pages=0, table_dev=None, k_dev=None)])
def test_a_cache_without_pages_or_a_table_without_entries_needs_no_memory(kw):
    """The checks get past the cache to what is refused behind it."""
    assert B.mdcnn_cache_attend_bytes(cache(**kw), attending(), 8, 1) == 0
    refused(4, B.mdcnn_cache_attend, cache(**kw), attending(), heads(heads=8, x_token=256, y_token=256), 1, FAKE + 2, None, 0)
    for call in (B.mdcnn_cache_store, B.mdcnn_cache_read):
        refused(1, call, cache(**kw), heads(), heads(), 3, None, FAKE, 3, 1)


def test_few_rows_of_many_long_sequences_go_by_the_tile():
    """32 to 64 rows of 64 sequences of 8192 tokens: tiles fill the GPU without splits, so nothing is left to be joined; two sequences are split, and so are rows of 32 channels."""
    def need(dim, n_seq, rows, dtype=1):
        c, a = cache(dim=dim, n_seq=n_seq, heads=8, max_pages=128, pages=9000), attending(tokens=n_seq * rows, max_new=rows, max_len=8192)
        return B.mdcnn_cache_attend_bytes(c, a, 8, dtype)
    assert need(128, 64, 48) == need(96, 64, 32) == need(128, 64, 64) == 0
    assert need(128, 2, 64) > 0 and need(32, 16, 64) > 0 and need(128, 16, 16) > 0 and need(128, 16, 64, 0) > 0
