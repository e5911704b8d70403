"""The oracle of the paged 8-bit cache against torch's conversion, hand-worked scales and plain attention (CPU)."""
import math

import numpy as np
import pytest
import torch

from oracle import page_oracle as O


def test_bytes_and_rounding_against_the_library_conversion():
    b = torch.arange(256, dtype=torch.uint8)
    ref = b.view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(np.isnan(ref), np.isnan(O.VALUES)) and np.array_equal(np.nan_to_num(ref), np.nan_to_num(O.VALUES))
    x = torch.cat([torch.linspace(-448, 448, 20011), torch.randn(5000) * 0.01, torch.tensor([0.0, -0.0, 2.0 ** -10, 1.5 * 2.0 ** -9, 17.0])])
    assert np.array_equal(O.encode(x.numpy()), x.to(torch.float8_e4m3fn).view(torch.uint8).numpy())
    assert O.encode(np.array([1e9, -np.inf, np.nan])).tolist() == [0x7E, 0xFE, 0x7F]


@pytest.mark.parametrize("top,exp", [(448.0, 0), (449.0, 1), (224.0, -1), (225.0, 0), (1.0, -8), (0.0, -60), (1.75, -8), (1.7578125, -7)])
def test_scale(top, exp):
    assert O.scale_exp(np.array([0.1 * top, -top, math.inf, math.nan])) == exp


def test_write_grows_a_scale_and_keeps_the_rest():
    k8, s = np.zeros((1, 2, 1, 16, 128), np.uint8), np.ones((1, 2, 1), np.float32)
    table = np.array([[1, 0]], np.int32)
    O.write(k8, s, 0, None, [3], [0, 3], None, np.full((3, 1, 128), 1.0), table)
    assert s[0, 1, 0] == 2.0 ** -8 and s[0, 0, 0] == 1.0 and k8[0, 1, 0, :3].min() == k8[0, 1, 0, :3].max() != 0 and not k8[0, 1, 0, 3:].any()
    O.write(k8, s, 0, None, [4], [0, 1], None, np.full((1, 1, 128), 4.0), table)
    assert s[0, 1, 0] == 2.0 ** -6 and np.all(O.values(k8, s, 0, 0, 4, table)[:3] == 1.0) and np.all(O.values(k8, s, 0, 0, 4, table)[3] == 4.0)
    O.write(k8, s, 0, None, [4], [0, 1], [3], np.full((1, 1, 128), 0.5), table)      # the others keep the scale up
    assert s[0, 1, 0] == 2.0 ** -6 and np.all(O.values(k8, s, 0, 0, 4, table)[3] == 0.5)


def test_attention_against_torch():
    rng = np.random.default_rng(3)
    q, k, v = rng.normal(size=(3, 4, 128)), rng.normal(size=(9, 2, 128)), rng.normal(size=(9, 2, 128))
    out, lse, _, _ = O.attn(q, k, v, 9)
    tq, tk, tv = (torch.from_numpy(x).transpose(0, 1) for x in (q, k, v))
    mask = torch.arange(9)[None] <= 6 + torch.arange(3)[:, None]
    z = tq @ tk.repeat_interleave(2, 0).transpose(1, 2) / math.sqrt(128)
    z = z.masked_fill(~mask, -math.inf)
    ref = (z.softmax(-1) @ tv.repeat_interleave(2, 0)).transpose(0, 1).numpy()
    assert np.abs(out - ref).max() < 1e-12 and np.abs(lse - z.logsumexp(-1).numpy()).max() < 1e-12


def test_fork_free_compact_by_hand():
    table, refs = np.full((4, 4), -1, np.int32), np.zeros(8, np.int32)
    data = np.arange(8.0).reshape(1, 8)
    p = O.Pool(table, refs, 16, [data])
    assert p.fork([-1], [0], [0], [40], True) == ""
    assert table[0].tolist() == [0, 1, 2, -1] and refs.tolist() == [1, 1, 1, 0, 0, 0, 0, 0]
    assert p.fork([0, 0], [1, 2], [40, 32], [50, 33], True) == ""
    assert table[1].tolist() == [0, 1, 3, 4] and table[2].tolist() == [0, 1, 5, -1] and data[0, 3] == 2.0
    assert refs.tolist() == [3, 3, 1, 1, 1, 1, 0, 0]
    assert p.fork([0], [3], [40], [64], False) == "pages" and table[3].tolist() == [-1] * 4
    p.free([0, 1], [0, 20])
    assert table[1].tolist() == [0, 1, -1, -1] and refs.tolist() == [2, 2, 0, 0, 0, 1, 0, 0]
    assert p.fork([2], [2], [20], [48], True) == ""          # page 1 is shared and only part of it kept
    assert table[2].tolist() == [0, 2, 5, -1] and refs.tolist() == [2, 1, 1, 0, 0, 1, 0, 0] and data[0, 2] == 1.0
    assert p.compact() == 4 and table[2].tolist() == [0, 2, 3, -1] and refs.tolist() == [2, 1, 1, 1, 0, 0, 0, 0] and data[0, 3] == 5.0


def test_growth_replaces_the_page_of_the_next_token_by_hand():
    table, refs = np.full((3, 3), -1, np.int32), np.zeros(4, np.int32)
    data = np.arange(4.0).reshape(1, 4)
    p = O.Pool(table, refs, 16, [data])
    assert p.fork([-1], [0], [0], [32], True) == "" and p.fork([0], [1], [32], [32], True) == ""
    assert p.fork([0], [0], [32], [32], True) == "" and table[0].tolist() == [0, 1, -1]       # its next token has no page yet
    assert p.fork([0], [0], [16], [32], True) == ""          # set back to a border: token 16 would go into row 1's page
    assert table.tolist() == [[0, 2, -1], [0, 1, -1], [-1] * 3] and refs.tolist() == [2, 1, 1, 0] and data[0, 2] == 1.0
    assert p.fork([0], [0], [16], [32], True) == "" and table[0].tolist() == [0, 2, -1]       # its own now
    assert p.fork([1], [1], [0], [1], True) == ""
    assert table[1].tolist() == [3, 1, -1] and refs.tolist() == [1, 1, 1, 1]
