"""What the operators on a step's rows refuse (CPU: every refusal comes from the
host's checks, before anything is enqueued; the addresses are never read)."""

import ctypes

import pytest

import paper_2606_01019_amd as hvd
from paper_2606_01019_amd import rows as R
from paper_2606_01019_amd.hvd import HVD_ERR_ARG, HVD_OK

A = 1 << 20  # an aligned address nothing dereferences


@pytest.fixture(scope="module")
def lib():
    return hvd.load_library()


def make(cls, base, kw):
    a = cls(**base)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def batch(**kw):
    return make(R.RowBatchC, dict(starts=A, lengths=A, pages=A, tree=A, pages_stride=8, n_seqs=3, max_pages=8), kw)


def kv(**kw):
    return make(R.PagedKVC, dict(k=A, k_page_stride=2 * 16 * 64, k_head_stride=16 * 64, k_token_stride=64, v=A,
                                 v_page_stride=2 * 16 * 64, v_head_stride=64, v_token_stride=128, n_pages=10, n_heads=2,
                                 page_size=16, head_dim=64, dtype=0), kw)


def append(**kw):
    return make(R.AppendArgs, dict(k=A, k_row_stride=512, k_head_stride=64, v=A, v_row_stride=512, v_head_stride=64, q=A,
                                   q_row_stride=512, q_head_stride=64, q_out=A, freqs=A, positions=A, q_heads=4, rot=64,
                                   interleaved=0, dtype=2), kw)


def attend(**kw):
    return make(R.AttendArgs, dict(q=A, q_row_stride=256, q_head_stride=64, out=A, out_row_stride=256, out_head_stride=64,
                                   slopes=A, first=A, prefix=A, scale=0.125, cap=30.0, q_heads=4, window=9), kw)


def adjust(**kw):
    return make(R.AdjustArgs, dict(logits=A, logits_stride=100, out=A, out_stride=100, best=A, tokens=A, history=A,
                                   history_stride=40, history_lengths=A, prompt_lengths=A, repetition=A, frequency=A,
                                   presence=A, bias_ids=A, bias_ids_stride=7, bias=A, bias_stride=7, allowed=A,
                                   allowed_stride=4, vocab=100, max_history=40, n_bias=7, dtype=2), kw)


ref = ctypes.byref
BAD_BATCH = [dict(starts=None), dict(starts=A + 2), dict(tree=A + 4), dict(n_seqs=-1), dict(n_seqs=4097)]
BAD_KEYS = [dict(lengths=None), dict(pages=None), dict(lengths=A + 1), dict(pages=A + 2), dict(pages_stride=7),
            dict(max_pages=-1), dict(max_pages=(1 << 25) + 1, pages_stride=1 << 26)]
BAD_KV = [dict(k=None), dict(v=None), dict(k=A + 8), dict(v=A + 2), dict(n_pages=-1), dict(n_heads=0), dict(n_heads=257),
          dict(page_size=8), dict(page_size=48), dict(page_size=2048), dict(head_dim=0), dict(head_dim=60),
          dict(head_dim=264), dict(dtype=2), dict(dtype=3), dict(dtype=-1), dict(k_page_stride=2047),
          dict(k_page_stride=1024), dict(k_token_stride=56), dict(v_head_stride=32), dict(v_token_stride=64),
          dict(k_token_stride=(1 << 26) + 8), dict(k_head_stride=-8), dict(v_page_stride=0), dict(k_page_stride=1 << 60)]


@pytest.mark.parametrize("kw", BAD_BATCH + BAD_KEYS)
def test_batch(lib, kw):
    b = batch(**kw)
    assert lib.hvd_append_kv(ref(b), ref(kv()), ref(append()), 4, None) == HVD_ERR_ARG
    assert lib.hvd_attend(ref(b), ref(kv()), ref(attend()), 4, A, 1 << 40, None) == HVD_ERR_ARG
    assert lib.hvd_attend_workspace(ref(b), ref(kv()), 4, 4) == 0
    if kw in BAD_BATCH:
        assert lib.hvd_adjust_logits(ref(b), ref(adjust()), 4, A, 1 << 40, None) == HVD_ERR_ARG
        assert lib.hvd_adjust_workspace(ref(b), ref(adjust()), 4) == 0
    assert lib.hvd_last_error()


@pytest.mark.parametrize("kw", BAD_KV)
def test_cache(lib, kw):
    assert lib.hvd_append_kv(ref(batch()), ref(kv(**kw)), ref(append()), 4, None) == HVD_ERR_ARG
    assert lib.hvd_attend(ref(batch()), ref(kv(**kw)), ref(attend()), 4, A, 1 << 40, None) == HVD_ERR_ARG
    assert lib.hvd_attend_workspace(ref(batch()), ref(kv(**kw)), 4, 4) == 0


@pytest.mark.parametrize("kw", [
    dict(k=None), dict(v=None), dict(k=A + 2), dict(v=A + 1), dict(q=A + 2), dict(q=None), dict(q_out=None),
    dict(q_out=A + 8), dict(freqs=None), dict(freqs=A + 4), dict(positions=A + 2), dict(q_heads=0), dict(q_heads=257),
    dict(rot=-2), dict(rot=63), dict(rot=66), dict(dtype=3), dict(dtype=-1), dict(k_row_stride=-1), dict(q_head_stride=-64)])
def test_append(lib, kw):
    assert lib.hvd_append_kv(ref(batch()), ref(kv()), ref(append(**kw)), 4, None) == HVD_ERR_ARG


@pytest.mark.parametrize("kw", [
    dict(q=None), dict(out=None), dict(q=A + 8), dict(out=A + 8), dict(q_row_stride=255), dict(q_head_stride=-64),
    dict(out_row_stride=100), dict(out_row_stride=56), dict(out_head_stride=56), dict(slopes=A + 2), dict(first=A + 1),
    dict(prefix=A + 3), dict(scale=float("nan")), dict(scale=float("inf")), dict(cap=-1.0), dict(cap=float("nan")),
    dict(cap=float("inf")), dict(window=-1), dict(q_heads=0), dict(q_heads=3), dict(q_heads=258)])
def test_attend(lib, kw):
    assert lib.hvd_attend(ref(batch()), ref(kv()), ref(attend(**kw)), 4, A, 1 << 40, None) == HVD_ERR_ARG


def test_attend_workspace(lib):
    n = lib.hvd_attend_workspace(ref(batch()), ref(kv()), 4, 4)
    assert n > 16
    for work, size in ((None, n), (A + 8, n), (A, n - 1)):
        assert lib.hvd_attend(ref(batch()), ref(kv()), ref(attend()), 4, work, size, None) == HVD_ERR_ARG
    assert lib.hvd_attend_workspace(ref(batch()), ref(kv()), 3, 4) == 0
    assert lib.hvd_attend_workspace(ref(batch()), ref(kv()), 4, -1) == 0
    assert lib.hvd_attend_workspace(ref(batch()), ref(kv()), 4, (1 << 20) + 1) == 0


@pytest.mark.parametrize("kw", [
    dict(logits=None), dict(out=None, best=None), dict(logits=A + 2), dict(out=A + 1), dict(best=A + 2), dict(tokens=A + 1),
    dict(history=A + 2), dict(history_lengths=None), dict(history_lengths=A + 2), dict(prompt_lengths=A + 1),
    dict(repetition=A + 2), dict(frequency=A + 2), dict(presence=A + 2), dict(bias=None), dict(bias_ids=None),
    dict(bias_ids=A + 2), dict(bias=A + 1), dict(allowed=A + 2), dict(vocab=0), dict(vocab=(1 << 24) + 1), dict(dtype=3),
    dict(logits_stride=99), dict(out_stride=99), dict(out_stride=101), dict(history_stride=39), dict(bias_stride=6),
    dict(bias_ids_stride=6), dict(allowed_stride=3), dict(max_history=-1), dict(max_history=983040), dict(n_bias=-1),
    dict(n_bias=2047)])
def test_adjust(lib, kw):
    assert lib.hvd_adjust_logits(ref(batch()), ref(adjust(**kw)), 4, A, 1 << 40, None) == HVD_ERR_ARG


def test_adjust_workspace(lib):
    n = lib.hvd_adjust_workspace(ref(batch()), ref(adjust()), 4)
    assert n >= 16
    for work, size in ((None, n), (A + 8, n), (A, 0)):
        assert lib.hvd_adjust_logits(ref(batch()), ref(adjust()), 4, work, size, None) == HVD_ERR_ARG
    assert lib.hvd_adjust_workspace(ref(batch()), ref(adjust()), 65537) == 0


def test_rows(lib):
    for rows in (-1, (1 << 20) + 1):
        assert lib.hvd_append_kv(ref(batch()), ref(kv()), ref(append()), rows, None) == HVD_ERR_ARG
        assert lib.hvd_attend(ref(batch()), ref(kv()), ref(attend()), rows, A, 1 << 40, None) == HVD_ERR_ARG
        assert lib.hvd_adjust_logits(ref(batch()), ref(adjust()), rows, A, 1 << 40, None) == HVD_ERR_ARG
    assert lib.hvd_append_kv(ref(batch()), ref(kv()), ref(append(k=None)), 0, None) == HVD_OK
    assert lib.hvd_attend(ref(batch()), ref(kv()), ref(attend(q=None)), 0, None, 0, None) == HVD_OK
    assert lib.hvd_adjust_logits(ref(batch()), ref(adjust(logits=None)), 0, None, 0, None) == HVD_OK
    assert lib.hvd_append_kv(None, ref(kv()), ref(append()), 0, None) == HVD_ERR_ARG
    assert lib.hvd_append_kv(ref(batch()), None, ref(append()), 0, None) == HVD_ERR_ARG
    assert lib.hvd_append_kv(ref(batch()), ref(kv()), None, 0, None) == HVD_ERR_ARG
    assert lib.hvd_attend(ref(batch()), ref(kv()), None, 0, A, 1 << 40, None) == HVD_ERR_ARG
    assert lib.hvd_adjust_logits(ref(batch()), None, 0, A, 1 << 40, None) == HVD_ERR_ARG


def test_tensors_on_the_host_are_refused():
    import torch
    z = torch.zeros(2, dtype=torch.int32)
    with pytest.raises(hvd.HvdError):
        hvd.RowBatch(z)
    with pytest.raises(hvd.HvdError):
        hvd.RowBatch([0, 1])
    for call in (lambda: hvd.attend(z, z, z, None), lambda: hvd.append_kv(z, z, z, z, "no batch"),
                 lambda: hvd.adjust_logits(z, None)):
        with pytest.raises(hvd.HvdError):
            call()


@pytest.mark.parametrize("kw", [
    dict(out_row_stride=64, out_head_stride=64),  # head 1 of a row is head 0 of the next one
    dict(out_row_stride=128, out_head_stride=64), dict(out_row_stride=64, out_head_stride=128),
    dict(out_row_stride=184, out_head_stride=64), dict(out_row_stride=1 << 60), dict(out_row_stride=0)])
def test_attend_places_of_out_that_meet(lib, kw):
    assert lib.hvd_attend(ref(batch()), ref(kv()), ref(attend(q=2 * A, **kw)), 4, A, 1 << 40, None) == HVD_ERR_ARG
    assert b"out overlap" in lib.hvd_last_error()


@pytest.mark.parametrize("kw", [
    dict(out_row_stride=512), dict(out_row_stride=64, out_head_stride=256),  # at q itself with other strides
    dict(out=A + 2 * 256), dict(out=A + 2 * 64), dict(out=A - 2 * 64), dict(out=A + 2 * (3 * 256 + 3 * 64)),
    dict(out=A - 2 * (3 * 256 + 3 * 64)), dict(out=A + 2 * 24), dict(out=A - 2 * 56),
    dict(q_row_stride=0), dict(q_row_stride=0, q_head_stride=0, out=A - 2 * (4 * 256 - 64)),
    dict(out=A + 2 * 256, q_row_stride=512, out_row_stride=512, q_head_stride=72, out_head_stride=72)])
def test_attend_out_that_shares_memory_with_q(lib, kw):
    assert lib.hvd_attend(ref(batch()), ref(kv()), ref(attend(**kw)), 4, A, 1 << 40, None) == HVD_ERR_ARG
    assert b"shares memory with q" in lib.hvd_last_error()


@pytest.mark.parametrize("kw", [
    dict(), dict(out=A + 2 * 4 * 256), dict(out=A - 2 * 4 * 256), dict(out=2 * A, out_row_stride=512),
    # beside q in one buffer: rows of [q, out], heads of [q, out]
    dict(out=A + 2 * 256, q_row_stride=512, out_row_stride=512), dict(out=A - 2 * 256, q_row_stride=512, out_row_stride=512),
    dict(out=A + 2 * 64, q_row_stride=512, q_head_stride=128, out_row_stride=512, out_head_stride=128),
    dict(out=A + 2 * 64, q_row_stride=128, q_head_stride=512, out_row_stride=128, out_head_stride=512),
    dict(out=A + 2 * 256, q_row_stride=0)])
def test_attend_out_that_has_its_own_memory(lib, kw):
    """Goes as far as the workspace's check, the last one."""
    assert lib.hvd_attend(ref(batch()), ref(kv()), ref(attend(**kw)), 4, None, 0, None) == HVD_ERR_ARG
    assert b"work must be" in lib.hvd_last_error()


@pytest.mark.parametrize("kw", [
    dict(out_stride=101), dict(out=A + 400), dict(out=A - 400), dict(out=A + 4), dict(out=A - 4 * 99),
    dict(out=A + 4 * 100, logits_stride=200, out_stride=300), dict(out=A + 4 * 99, logits_stride=200, out_stride=200),
    dict(dtype=0, out=A + 2), dict(dtype=1, out=A - 2 * 399)])
def test_adjust_out_that_shares_memory_with_logits(lib, kw):
    assert lib.hvd_adjust_logits(ref(batch()), ref(adjust(**kw)), 4, A, 1 << 40, None) == HVD_ERR_ARG
    assert b"shares memory with logits" in lib.hvd_last_error()


@pytest.mark.parametrize("kw", [
    dict(), dict(out=None), dict(out=A + 1600), dict(out=A - 1600), dict(out=A + 400, logits_stride=200, out_stride=200),
    dict(out=A - 400, logits_stride=200, out_stride=200), dict(dtype=0, out=A + 800)])
def test_adjust_out_that_has_its_own_memory(lib, kw):
    """Goes as far as the workspace's check, the last one."""
    assert lib.hvd_adjust_logits(ref(batch()), ref(adjust(**kw)), 4, None, 0, None) == HVD_ERR_ARG
    assert b"work must be" in lib.hvd_last_error()


SAME = dict(v_head_stride=1024, v_token_stride=64)  # the strides of k


@pytest.mark.parametrize("kw", [
    dict(), SAME, dict(SAME, v=A + 2 * 64), dict(SAME, v=A - 2 * 9 * 2048), dict(SAME, v=A + 2 * (9 * 2048 + 1024 + 15 * 64)),
    dict(SAME, v=A + 2 * 32, k_token_stride=64, k_head_stride=2048, k_page_stride=4096, v_head_stride=2048, v_page_stride=4096),
    dict(v=A + 2 * 1024, k_page_stride=4096, v_page_stride=4096)])
def test_append_keys_and_values_that_share_memory(lib, kw):
    assert lib.hvd_append_kv(ref(batch()), ref(kv(**kw)), ref(append()), 4, None) == HVD_ERR_ARG
    assert b"share memory" in lib.hvd_last_error()


@pytest.mark.parametrize("scale", [1.8e38, -1.8e38, 3.4e38, 2.4e38, float("-inf")])
def test_attend_a_scale_whose_exponents_have_no_factor(lib, scale):
    """scale log2 e is infinite from 2.36e38 on."""
    assert lib.hvd_attend(ref(batch()), ref(kv()), ref(attend(scale=scale)), 4, A, 1 << 40, None) == HVD_ERR_ARG
    assert b"scale" in lib.hvd_last_error()
