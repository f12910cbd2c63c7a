"""The received weight on each of its kernels: K streamed for up to 16 and up to 64 rows of a (sequence, KV
head), blocks of 32 and of 128 keys for more, for every type, head size and page."""
import numpy as np
import pytest
import torch

from tests import cache_ref as R
from tests.gpu_helpers import log
from tests.test_gpu_cache import cu_of, dev, dev_cache, within

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def A():
    from paper_2606_06521_amd import attn_fp8
    return attn_fp8


# most rows of a (sequence, KV head), tokens that the table has room for, new tokens, lens; two KV heads
KERNELS = {
    "stream16": (16, 1024, [4, 1, 0], [900, 70, 5]), "stream64": (64, 1024, [16, 5, 11], [901, 64, 11]),
    "keys32": (10 ** 6, 1024, [70, 40, 1], [700, 40, 129]), "keys128": (10 ** 6, 6016, [70, 40, 17], [1200, 300, 17]),
}


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("kernel", KERNELS)
@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("d,page", [(64, 64), (64, 128), (128, 64), (128, 128)])
def test_every_kernel(A, d, page, kind, kernel, causal):
    G, Hkv, B = 4, 2, 3
    most, room, new, lens = KERNELS[kernel]
    n_cu = torch.cuda.get_device_properties(0).multi_processor_count
    rows, visits = max(new) * G, -(-room // 128)
    assert rows <= most and (kernel.startswith("stream") or rows > 64) and (kernel != "stream64" or rows > 16)
    assert not kernel.startswith("keys") or n_cu != 256 or (B * Hkv * visits < n_cu) == (kernel == "keys32")
    rng = np.random.default_rng(room + d + page)
    c = R.make_cache(rng, B, Hkv, page, d, lens, W=-(-room // page))
    c.pages[0, 2] = -1                                    # no page: nobody sees its keys, their entries stay
    T, cu, n_w = sum(new), cu_of(new), c.pages.shape[1] * page
    q = R.make_queries(rng, T, G * Hkv, d)
    lse = R.attention(c, q, G, cu=cu, causal=causal)[1].astype(np.float32)
    lse[T // 2, 1] = -np.inf                              # a row that adds nothing
    start = rng.random((B, Hkv, n_w + 3)).astype(np.float32)
    w = dev(start)
    wide = torch.zeros((T, G * Hkv + 3, d), dtype=torch.bfloat16 if kind == "bf16" else torch.uint8, device="cuda")
    gq = R.torch_q(q, kind).cuda()
    wide[:, 2:G * Hkv + 2] = gq if kind == "bf16" else gq.view(torch.uint8)
    view = wide[:, 2:G * Hkv + 2]
    log(f"weights {kernel} d={d} page={page} {kind} causal={causal}")
    A.cache_weights(view if kind == "bf16" else view.view(torch.float8_e4m3fn), dev(lse), dev_cache(A, c), dev(c.pages), dev(c.lens),
                    w, cu=dev(cu), max_q=max(new), causal=causal)
    want = R.weights(c, q, lse, G, n_w + 3, cu=cu, causal=causal)
    got = w.cpu().double().numpy()
    # as in test_gpu_cache: 2^-17 of what is added (cache_ref), the sum's own rounding
    within(got, start + want, 2.0 ** -17 * want + 2.0 ** -24 * (start + want))
    assert np.array_equal(got[want == 0], start[want == 0].astype(np.float64))


@pytest.mark.parametrize("kernel", KERNELS)
def test_bound_on_the_length(A, kernel):
    """Entries from max_len on stay, whatever lens says."""
    G, Hkv, B, d, page = 4, 2, 3, 128, 64
    _, _, new, lens = KERNELS[kernel]
    rng = np.random.default_rng(d)
    c = R.make_cache(rng, B, Hkv, page, d, lens)
    T, cu, n_w = sum(new), cu_of(new), c.pages.shape[1] * page
    q = R.make_queries(rng, T, G * Hkv, d)
    lse = R.attention(c, q, G, cu=cu)[1].astype(np.float32)
    cut = max(lens) - max(new) - 35
    w = torch.zeros((B, Hkv, cut), device="cuda")
    log(f"weights {kernel} max_len={cut}")
    A.cache_weights(R.torch_q(q, "bf16").cuda(), dev(lse), dev_cache(A, c), dev(c.pages), dev(c.lens), w, cu=dev(cu), max_q=max(new),
                    max_len=cut)
    want = R.weights(c, q, lse, G, n_w, cu=cu)[:, :, :cut]
    within(w.cpu().double().numpy(), want, 2.0 ** -17 * want)


@pytest.mark.parametrize("max_q", [1 << 16, 1 << 22])
def test_a_loose_bound_on_the_new_tokens(A, max_q):
    """The weights' launch does not grow with max_q."""
    G, Hkv, B, d, page = 4, 8, 64, 64, 64
    rng = np.random.default_rng(5)
    lens, new = [int(n) for n in rng.integers(1, 100, B)], [1] * B
    c = R.make_cache(rng, B, Hkv, page, d, lens)
    q = R.make_queries(rng, B, G * Hkv, d)
    lse = R.attention(c, q, G, cu=cu_of(new))[1].astype(np.float32)
    n_w = c.pages.shape[1] * page
    w = torch.zeros((B, Hkv, n_w), device="cuda")
    log(f"weights max_q={max_q}")
    A.cache_weights(R.torch_q(q, "bf16").cuda(), dev(lse), dev_cache(A, c), dev(c.pages), dev(c.lens), w, cu=dev(cu_of(new)), max_q=max_q)
    want = R.weights(c, q, lse, G, n_w, cu=cu_of(new))
    within(w.cpu().double().numpy(), want, 2.0 ** -17 * want)
