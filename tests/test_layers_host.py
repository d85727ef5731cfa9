"""CPU tests of the operators of a decoder's layers: the list of sequences, which tiles the attention
kernels make of it, and what the host side refuses before it reaches the GPU."""

import ctypes

import numpy as np
import pytest

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def M():
    import __graft_entry__
    __graft_entry__.build()
    import paper_2609_15037_gb300 as pkg
    return pkg


def plan(M, lengths):
    size = M.moara_sequences_bytes(lengths)
    buf = np.full(max(1, size // 4) + 4, -7, dtype=np.int32)
    d = M.moara_sequences_init(lengths, buf.ctypes.data, size)
    assert (buf[size // 4:] == -7).all()
    rows = buf[:size // 4].reshape(-1, 4)
    return d, rows[:d.n_pairs], rows[d.n_pairs:]


def place(entries, n, heads, rows):
    """Entry n of a list of heads times its tiles, as the kernels read it."""
    begin, length, first, _ = (int(x) for x in entries[n // heads])
    tiles = (length - 1) // rows + 1
    most = max(1, min(heads, 304 // tiles))
    r = n - first * heads
    group = r // (most * tiles)
    have = min(most, heads - group * most)
    r -= group * most * tiles
    return begin, length, r // have, group * most + r % have


LENGTHS = [[1], [128], [129], [0, 5, 0, 300, 128], [1000, 1, 1000, 257, 0], [4096] * 3, [40000, 7]]


@pytest.mark.parametrize("heads", [1, 4, 7, 32])
@pytest.mark.parametrize("lengths", LENGTHS, ids=lambda x: "-".join(map(str, x)))
def test_every_tile_of_every_head_once(M, lengths, heads):
    d, pairs, tiles = plan(M, lengths)
    n = [-(-x // 128) for x in lengths]
    assert d.tokens == sum(lengths) and d.n_tiles == len(tiles) == sum(n) and d.n_pairs == len(pairs) == sum(-(-x // 256) for x in lengths)
    assert d.longest == max(n) and d.work == sum(x * (x + 1) // 2 for x in n)
    begins = np.concatenate([[0], np.cumsum(lengths)[:-1]])
    for entries, rows in ((pairs, 256), (tiles, 128)):
        want = {(int(b), x, t, h) for b, x in zip(begins, lengths) for t in range(-(-x // rows)) for h in range(heads)}
        got = [place(entries, i, heads, rows) for i in range(len(entries) * heads)]
        assert len(got) == len(want) and set(got) == want
        assert all(a >= b for a, b in zip(entries[:, 1], entries[1:, 1]))      # the longest sequences first


def test_no_sequences(M):
    for lengths in ([], [0], [0, 0, 0]):
        d, pairs, tiles = plan(M, lengths)
        assert (d.tokens, d.n_tiles, d.n_pairs, d.longest, d.work) == (0, 0, 0, 0, 0)


def test_lengths_are_refused(M):
    for lengths in ([-1], [5, -2], [2 ** 31 - 1], [2 ** 30, 2 ** 30]):
        with pytest.raises(M.MoaraError) as e:
            M.moara_sequences_bytes(lengths)
        assert e.value.code == M.MOARA_ERR_SHAPE
    for lengths in ([2 ** 31], [3, 2 ** 40]):
        with pytest.raises(ValueError):
            M.moara_sequences_bytes(lengths)
    lib = M.binding.lib
    out = M.binding.moara_sequences()
    one = (ctypes.c_int * 1)(300)
    assert lib.moara_sequences_init(1, one, None, 0, ctypes.byref(out)) == M.MOARA_ERR_WORKSPACE
    assert lib.moara_sequences_init(1, None, None, 0, ctypes.byref(out)) == M.MOARA_ERR_INVALID_ARG
    assert lib.moara_sequences_init(-1, one, None, 0, ctypes.byref(out)) == M.MOARA_ERR_INVALID_ARG
    assert lib.moara_sequences_init(1, one, None, 0, None) == M.MOARA_ERR_INVALID_ARG
    assert lib.moara_sequences_bytes(1, one, None) == M.MOARA_ERR_INVALID_ARG


def test_struct_matches_header(M):
    s = M.binding.moara_sequences
    assert ctypes.sizeof(s) == 32 and s.tokens.offset == 8 and s.longest.offset == 20 and s.work.offset == 24


def test_null_context_is_refused(M):
    lib = M.binding.lib
    bad = M.MOARA_ERR_INVALID_ARG
    assert lib.moara_rms_norm(None, 1, 1, None, 1, None, 1, 0, None, 0.0, None, 1, None, 0, 1, None, None) == bad
    assert lib.moara_rms_norm_quantize(None, 1, 1, None, 1, None, 1, 0, None, 0.0, None, 1, None, None, None, None, None, None) == bad
    assert lib.moara_rms_norm_backward(None, 1, 1, None, 0, 1, None, 0, 1, None, None, None, 1, None, 1, None, None, 0, None) == bad
    assert lib.moara_attention(None, None, 1, 1, 1, 64, 1.0, None, 0, 0, None, 0, 0, None, 0, 0, None, None, None, None) == bad
    assert lib.moara_policy_loss(None, 1, 1, None, 0, 1, None, None, None, None, None, 0.8, 1.2, 0.0, None, None, None, 1, None, 0,
                                 None) == bad


def test_workspaces(M):
    assert M.moara_rms_norm_backward_workspace_bytes(1, 1) >= 4
    for rows, cols in ((1, 49152), (16384, 4096), (300, 33), (10 ** 6, 16), (5000, 4099)):
        size = M.moara_rms_norm_backward_workspace_bytes(rows, cols)
        assert size % (4 * cols) == 0 and size <= 152 * 16 * cols * 4
    assert M.moara_policy_loss_workspace_bytes(1) == 24 and M.moara_policy_loss_workspace_bytes(10 ** 8) == 152 * 16 * 24
    for call, code in ((lambda: M.moara_rms_norm_backward_workspace_bytes(0, 1), M.MOARA_ERR_SHAPE),
                       (lambda: M.moara_rms_norm_backward_workspace_bytes(1, 49153), M.MOARA_ERR_UNSUPPORTED),
                       (lambda: M.moara_policy_loss_workspace_bytes(0), M.MOARA_ERR_SHAPE)):
        with pytest.raises(M.MoaraError) as e:
            call()
        assert e.value.code == code


@pytest.mark.parametrize("big", [2 ** 31, -2 ** 32 + 1])
def test_sizes_beyond_32_bits_are_refused(M, big):
    seqs = M.binding.moara_sequences()
    for call in (lambda: M.moara_rms_norm_backward_workspace_bytes(big, 1), lambda: M.moara_policy_loss_workspace_bytes(big),
                 lambda: M.moara_rms_norm(None, big, 1, 0, 1, 0, 1, 0, 0, 0.0, 0, 1, 0, 0, 1, 0),
                 lambda: M.moara_attention(None, seqs, big, 1, 1, 64, 1.0, *[0] * 12),
                 lambda: M.moara_policy_loss(None, 1, big, 0, 0, 1, 0, 0, 0, 0, 0, 0.8, 1.2, 0.0, 0, 0, 0, 1, 0, 0)):
        with pytest.raises(ValueError):
            call()


def group(M, device=0):
    g = M.LayerGroup.__new__(M.LayerGroup)
    g.device, g.ctx = device, 0
    return g


def test_sequences_of_another_device_are_refused(M):
    s = M.Sequences.__new__(M.Sequences)
    s.device = 1
    x = torch.zeros(4, 2, 64, dtype=torch.bfloat16)
    for call in (lambda: group(M).attention(x, x, x, s), lambda: group(M).attention_backward(x, x, x, x, x, x, s)):
        with pytest.raises(ValueError):
            call()


def test_tensors_of_the_host_are_refused(M, monkeypatch):
    """Before any entry is called."""
    g = group(M)
    for name in ("_NORM", "_NORM_QUANTIZE", "_NORM_BACKWARD", "_ATTENTION", "_LOSS"):
        monkeypatch.setattr(M.layers, name, 0)               # a call would end the process
    monkeypatch.setattr(M.layers, "stream_handle", lambda s, d: 0)
    x, v = torch.zeros(4, 8), torch.zeros(8)
    for call in (lambda: g.norm(x, v), lambda: g.norm_quantize(x, v), lambda: g.norm_backward(x, x, v, torch.zeros(4)),
                 lambda: g.policy_loss(x, torch.zeros(4, dtype=torch.int64), *[torch.zeros(4)] * 2),
                 lambda: g.norm(None, v), lambda: g.norm_quantize(x, v, rows=False), lambda: g.norm(x, v, dtype=torch.float16),
                 lambda: g.policy_loss(x, torch.zeros(4, dtype=torch.int64), *[torch.zeros(4)] * 2, kl=0.1)):
        with pytest.raises(ValueError):
            call()
