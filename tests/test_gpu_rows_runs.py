"""Alternatives of rows that a mask holds to a run of tokens, and of rows whose last part is short: right, and about as
fast as those of other rows."""
import numpy as np
import pytest
import torch

import util_rows as ur
from test_gpu_logprobs import check_logprobs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n_top", [8, 20, 32, 33, 128])
@pytest.mark.parametrize("n,v", [(2, 600), (2, 12000), (2, 50257), (2, 151936), (260, 20000)])
def test_runs_of_every_length(n, v, n_top, dtype):
    """Runs of 1 to 3,000 tokens anywhere, of different, equal and few different logits."""
    print(f"[case] {n}x{v} {dtype} top {n_top}", flush=True)
    rng = np.random.default_rng([n, v, n_top])
    rows = []
    for i, m in enumerate((1, 7, 19, 20, 64, 127, 150, 256, 300, 500, 1000, 1017, 3000)):
        for kind in range(3):
            m = min(m, v)
            x = np.full(v, -np.inf if (i + kind) % 2 else np.nan, np.float32)
            at = int(rng.integers(0, v - m + 1))
            x[at:at + m] = (rng.standard_normal(m) * 3, 1.5, rng.integers(0, 3, m))[kind]
            rows.append(x)
    x = np.array(rows)
    x = np.tile(x, (-(-n // len(x)), 1))
    check_logprobs(x, ur.placed(x, dtype, pad=1), rng.integers(0, v, len(x)), None, n_top)


def gpu_time(rows, n_top, reps=10):
    """us of the GPU for a call, the least of five replays of a graph of several."""
    import paper_2510_15545_amd as tt

    call = lambda: tt.logprobs(rows.shape[1], rows, n_top=n_top)  # noqa: E731
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for _ in range(reps):
            call()
    best = float("inf")
    for _ in range(6):
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        a.record()
        graph.replay()
        b.record()
        torch.cuda.synchronize()
        best = min(best, a.elapsed_time(b) * 1e3 / reps)
    return best


@pytest.mark.parametrize("n,v,n_top,m", [(1, 151936, 20, 256), (1, 151936, 32, 500), (48, 128256, 20, 300), (1, 50257, 20, 500), (64, 50257, 32, 1000)])
def test_a_run_takes_no_longer(n, v, n_top, m):
    """Every element read again 57 times, one by one, would take 15 to 30 times as long."""
    x = torch.randn((n, v), device="cuda", generator=torch.Generator(device="cuda").manual_seed(1)).mul_(3).bfloat16()
    ordinary = gpu_time(x, n_top)
    x[:, :v // 3] = -float("inf")
    x[:, v // 3 + m:] = -float("inf")
    run = gpu_time(x, n_top)
    print(f"[time] {n}x{v} top {n_top}: {ordinary:.1f} us, a run of {m}: {run:.1f}", flush=True)
    assert run <= 4 * ordinary


@pytest.mark.parametrize("n", [1, 48])
def test_parts_with_few_or_many_keys_take_no_longer(n):
    """A short last part, and as many alternatives as take the joining kernel to the keys it can hold."""
    gen = torch.Generator(device="cuda").manual_seed(1)
    x = {v: torch.randn((n, v), device="cuda", generator=gen).mul_(3).bfloat16() for v in (151936, 147856, 147556)}
    ordinary = gpu_time(x[151936], 20)
    for n_top in (20, 28, 31, 32, 33):
        for v, rows in x.items():
            us = gpu_time(rows, n_top)
            print(f"[time] {n}x{v} top {n_top}: {us:.1f} us", flush=True)
            assert us <= 2 * ordinary


def spoilt(rng, v):
    """Rows whose likely tokens come late: their first part masked, low or rising, by minus infinity, NaN or -30."""
    rows = []
    for share in (0.1, 0.35, 0.51, 0.7, 0.95):
        for low in (-np.inf, np.nan, -30.0):
            x = (rng.standard_normal(v) * 3).astype(np.float32)
            x[:int(v * share)] = low
            rows.append(x)
    at = np.arange(v, dtype=np.float32)
    rows += [at / v * 20, -at / v * 20, at / v * 20 + rng.standard_normal(v).astype(np.float32), np.where(at > v // 2, 5.0, at / v).astype(np.float32)]
    return np.array(rows, np.float32)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n_top", [1, 20, 32, 33, 128])
@pytest.mark.parametrize("n,v", [(1, 9001), (1, 20011), (1, 50257), (260, 30011), (1, 200003), (500, 50257)])
def test_likely_tokens_late_in_the_row(n, v, n_top, dtype):
    print(f"[case] {n}x{v} {dtype} top {n_top}", flush=True)
    rng = np.random.default_rng([n, v, n_top])
    x = spoilt(rng, v)
    rows = ur.placed(x, dtype, pad=1).repeat(-(-n // len(x)), 1)[:, :v]
    got = tt_logprobs(rows, n_top)
    for a in range(0, len(rows), len(x)):  # every copy of them has the first one's (sums' last digits go by alignment)
        assert torch.equal(got.top_ids[a:a + len(x)], got.top_ids[:len(x)])
    check_logprobs(x, rows[:len(x)], rng.integers(0, v, len(x)), None, n_top)
    want = ur.logprobs(ur.host(rows[:len(x)]), None, None, n_top)
    assert np.array_equal(got.top_ids[:len(x)].cpu().numpy(), want["top_ids"])


def tt_logprobs(rows, n_top):
    import paper_2510_15545_amd as tt

    return tt.logprobs(rows.shape[1], rows, n_top=n_top)


@pytest.mark.parametrize("n,v,n_top", [(1, 65536, 20), (64, 50257, 32), (300, 128256, 20), (512, 262144, 64), (40, 1000000, 20)])
def test_likely_tokens_late_in_the_row_take_no_longer(n, v, n_top):
    """A row's second reading at most, not 57 of them."""
    x = torch.randn((n, v), device="cuda", generator=torch.Generator(device="cuda").manual_seed(1)).mul_(3).bfloat16()
    ordinary = gpu_time(x, n_top)
    for share in (0.2, 0.51, 0.7):
        x[:, :int(v * share)] = -float("inf")
        late = gpu_time(x, n_top, 3)
        print(f"[time] {n}x{v} top {n_top}: {ordinary:.1f} us, the first {share} masked: {late:.1f}", flush=True)
        assert late <= 6 * ordinary
    rising = gpu_time((torch.arange(v, device="cuda") / v * 20).bfloat16().expand(n, v).contiguous(), n_top, 3)
    print(f"[time] {n}x{v} top {n_top}: {ordinary:.1f} us, rising: {rising:.1f}", flush=True)
    assert rising <= 6 * ordinary


@pytest.mark.parametrize("n,v,n_top", [(1, 151936, 64), (48, 151936, 64), (48, 128256, 128), (9, 300007, 128), (90, 262144, 100)])
def test_rows_of_equal_logits_take_no_longer(n, v, n_top):
    """Rows of zeros (a padded batch), of two values, and rows that rise by steps, of which every part hands over n_top."""
    x = torch.randn((n, v), device="cuda", generator=torch.Generator(device="cuda").manual_seed(1)).mul_(3).bfloat16()
    ordinary = gpu_time(x, n_top)
    at = torch.arange(v, device="cuda")
    for name, row in (("zeros", at * 0.0), ("two values", at % 3 // 2 * 1.0), ("steps", at // 1000 * 0.125)):
        x.copy_(row)
        us = gpu_time(x, n_top, 3)
        print(f"[time] {n}x{v} top {n_top}: {ordinary:.1f} us, {name}: {us:.1f}", flush=True)
        assert us <= 8 * ordinary  # 24 to 41 times as long by 64 searches
        want = torch.sort(x[0].float(), descending=True, stable=True).indices[:n_top].int()
        assert torch.equal(tt_logprobs(x, n_top).top_ids, want.expand(n, n_top))
