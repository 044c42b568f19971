"""Attention over the 4-bit cache where its inputs are far apart in size, or are no numbers: single
queries and drafts as well as chunks that are attended to on the tensor cores, with the same answers.

The bounds are those of test_kv4.py; what a row does not see leaves no trace in it.
"""
import os
import subprocess
import sys

import numpy as np
import pytest

import ops_reference as R
import paper_2606_07713_gb300 as pkg
from paper_2606_07713_gb300 import _lib
from test_kv4 import cast, check, dev, host, table_of
from test_kv4_chunks import reference, widened

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

HQ, HK, PAGE = 4, 1, 64
ROWS = [1, 40, 512]      # 4, 160 and 2048 query rows of the key head: the last as a chunk


def filled(k, v):
    """A pool holding keys and values [1, H, T, d] in shuffled pages, and its table."""
    table, n_pages = table_of(np.random.default_rng(1), [k.shape[2]], PAGE)
    pool = torch.full((n_pages, HK, PAGE // 16, 9 * (k.shape[3] + v.shape[3])), 255, dtype=torch.uint8, device="cuda:0")
    pos = np.arange(k.shape[2], dtype=np.int32)[None]
    pkg.kv4_write(dev(k, "bf16"), dev(v, "bf16"), pool, dev(table), dev(pos))
    return pool, dev(table)


def attend(q, k, v, causal=True):
    o, lse = pkg.kv4_attn_lse(dev(q, "bf16"), *filled(k, v), dev(np.array([k.shape[2]], dtype=np.int32)),
                              max_len=k.shape[2], causal=causal)
    assert pkg.get_device_status() == _lib.MOA_OK
    return o, lse


def inputs(N, T, dk, dv, seed):
    if N == 512:
        assert widened(1, HQ, HK, N, dk, dv, T)
    r = np.random.default_rng(seed)
    q = r.normal(size=(1, HQ, N, dk))
    return q, r.normal(size=(1, HK, T, dk)), r.normal(size=(1, HK, T, dv))


def stored(k, v):
    return R.values(*R.quantise(k)), R.values(*R.quantise(v))


@pytest.mark.parametrize("power", [20, 28, 30, 36, 60, 100])
@pytest.mark.parametrize("N", ROWS)
def test_keys_of_mixed_sizes(N, power):
    """Every third token's keys, and 32 features of every other token's, are 2^power times larger than the
    rest, where the queries are zero: the scores are those of the small ones."""
    T, d = 4100, 128
    q, k, v = inputs(N, T, d, d, seed=power)
    q[..., 32:64] = 0.0
    third = np.arange(T) % 3 == 0
    k[:, :, ~third & (np.arange(T) % 2 == 1), 32:64] *= 2.0 ** power
    k[:, :, third, :32] = k[:, :, third, 64:] = 0.0
    k[:, :, third, 32:64] *= 2.0 ** (power - 3)
    q, k, v = cast(q, "bf16"), cast(k, "bf16"), cast(v, "bf16")
    o, lse = attend(q, k, v)
    check(o, lse, reference(q, *stored(k, v), [T], d ** -0.5, True), d, "bf16", power)


@pytest.mark.parametrize("power", [20, 40, 100])
@pytest.mark.parametrize("d", [64, 128])
def test_a_huge_key_is_no_concern_of_rows_before_it(d, power):
    N, T, at = 512, 4096, 3800
    q, k, v = inputs(N, T, d, d, seed=power + d)
    k[:, :, at] *= 2.0 ** power
    q, k, v = cast(q, "bf16"), cast(k, "bf16"), cast(v, "bf16")
    before = at - (T - N)                     # rows that do not see it
    o, lse = attend(q, k, v)
    ref = reference(q, *stored(k, v), [T], d ** -0.5, True)
    check(o[:, :, :before], lse[:, :, :before], [x[:, :, :before] for x in ref], d, "bf16", power)


def test_single_precision_reads_of_mixed_sizes():
    """The cache itself loses nothing of them: what the cases above expect is what it holds."""
    T, d = 64, 128
    _, k, v = inputs(1, T, d, d, seed=8)
    k[:, :, ::2, 32:64] *= 2.0 ** 100
    k, v = cast(k, "bf16"), cast(v, "bf16")
    pool, table = filled(k, v)
    got = pkg.kv4_read(pool, table, dev(np.arange(T, dtype=np.int32)[None]), d, dtype=torch.float32)
    for x, y in zip(got, stored(k, v)):
        assert np.array_equal(host(x), y)
@pytest.mark.parametrize("dv", [64, 128])
@pytest.mark.parametrize("N", ROWS)
def test_a_value_that_is_no_number_reaches_its_group_only(N, dv):
    """The rows that see it are NaN in the 32 features of its group, however small its weight; the other
    features, the other rows and every log-sum-exp keep their bits."""
    T, d = 4000, 64
    q, k, v = inputs(N, T, d, dv, seed=dv)
    token = T - 1 - N // 2
    q[..., 0] = 1.0
    k[:, :, token] = 0.0
    k[:, :, token, 0] = -4096.0               # its weight is e^-512: nothing in 32 bits
    q, k, v = cast(q, "bf16"), cast(k, "bf16"), cast(v, "bf16")
    good, good_lse = attend(q, k, v)
    v[:, :, token, 33] = np.inf
    o, lse = attend(q, k, v)
    first = N - 1 - N // 2                    # the first row that sees it
    assert bool(torch.isnan(o[:, :, first:, 32:64]).all())
    o[:, :, first:, 32:64] = good[:, :, first:, 32:64]
    assert torch.equal(o, good) and torch.equal(lse, good_lse)


@pytest.mark.parametrize("N", ROWS)
def test_an_infinite_query_gives_nan(N):
    """Scores of minus infinity for every visible token have no softmax: NaN, not an empty row."""
    T, d = 4000, 64
    q, k, v = inputs(N, T, d, d, seed=3)
    k[..., 5] = -1.0 - np.abs(k[..., 5])
    q, k, v = cast(q, "bf16"), cast(k, "bf16"), cast(v, "bf16")
    good, good_lse = attend(q, k, v)
    q[0, 2, N - 1] = 0.0
    q[0, 2, N - 1, 5] = np.inf
    o, lse = attend(q, k, v)
    assert bool(torch.isnan(o[0, 2, N - 1]).all()) and bool(torch.isnan(lse[0, 2, N - 1]))
    o[0, 2, N - 1], lse[0, 2, N - 1] = good[0, 2, N - 1], good_lse[0, 2, N - 1]
    assert torch.equal(o, good) and torch.equal(lse, good_lse)


@pytest.mark.parametrize("N", [40, 512])
def test_the_largest_values_are_no_concern_of_rows_before_them(N):
    T, d = 4000, 64
    q, k, v = inputs(N, T, d, d, seed=4)
    q, k, v = cast(q, "bf16"), cast(k, "bf16"), cast(v, "bf16")
    good, _ = attend(q, k, v)
    token = T - 1 - N // 2
    v[:, :, token] = 3.3895313892515355e38    # the largest bf16
    o, _ = attend(q, k, v)
    first = N - 1 - N // 2
    assert torch.equal(o[:, :, :first], good[:, :, :first])




def test_slow_items_do_not_run_out_of_time():
    """Chunks all of whose tiles take the slow path keep within the kernel's time limits, which are per wait:
    here 5 ms each, read once a process, while an item takes about 40 ms."""
    code = (
        "import torch, paper_2606_07713_gb300 as p\n"
        "L, H, d, N, page = 16384, 8, 128, 2048, 64\n"
        "pool = p.kv4_pool(L // page, H, page, d, d)\n"
        "pages = torch.arange(L // page, dtype=torch.int32, device='cuda')[None]\n"
        "k = torch.randn(1, H, L, d, device='cuda')\n"
        "k[:, :, ::100, 32:64] *= 2.0 ** 30\n"
        "v = torch.randn(1, H, L, d, device='cuda').bfloat16()\n"
        "p.kv4_write(k.bfloat16(), v, pool, pages, torch.arange(L, dtype=torch.int32, device='cuda')[None])\n"
        "q = torch.randn(1, 4 * H, N, d, device='cuda').bfloat16()\n"
        "p.kv4_attn(q, pool, pages, torch.tensor([L], dtype=torch.int32, device='cuda'))\n"
        "print('status', p.get_device_status())\n")
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=300,
                       env=dict(os.environ, MOA_WAIT_LIMIT_NS="5000000", PYTHONPATH=root))
    assert r.returncode == 0 and "status 0" in r.stdout, r.stdout + r.stderr


@pytest.mark.parametrize("N", [1, 4, 40])
def test_single_precision_queries(N):
    """The fp32 form: a value that is no number and hardly weighs, and an infinite query."""
    T, d = 1003, 64
    q, k, v = inputs(N, T, d, d, seed=21)
    token = T - 1 - N // 2
    q[..., 0], k[:, :, token], k[:, :, token, 0] = 1.0, 0.0, -4096.0
    q, k, v = (cast(x, "fp32") for x in (q, k, v))

    def run(q, v):
        o, lse = pkg.kv4_attn_lse(dev(q, "fp32"), *filled(k, v), dev(np.array([T], dtype=np.int32)), max_len=T)
        assert pkg.get_device_status() == _lib.MOA_OK
        return o, lse

    good, good_lse = run(q, v)
    w, x = v.copy(), q.copy()
    w[:, :, token, 33] = np.nan
    o, lse = run(q, w)
    first = N - 1 - N // 2
    assert bool(torch.isnan(o[:, :, first:, 32:64]).all())
    o[:, :, first:, 32:64] = good[:, :, first:, 32:64]
    assert torch.equal(o, good) and torch.equal(lse, good_lse)
    x[0, 1, 0, 7] = -np.inf
    o, lse = run(x, v)
    assert bool(torch.isnan(o[0, 1, 0]).all()) and bool(torch.isnan(lse[0, 1, 0]))
    o[0, 1, 0], lse[0, 1, 0] = good[0, 1, 0], good_lse[0, 1, 0]
    assert torch.equal(o, good) and torch.equal(lse, good_lse)
