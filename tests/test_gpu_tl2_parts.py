"""The 1.78-bit layout's product taken apart, at sizes on both sides of the 4 MiB from which a launch streams its weights: codes against the oracle's, the
weights that come back, accumulators from codes and activations as the device holds them, and the same launch again.  A mismatch says which rows differ, by
how much, and in which part."""
import numpy as np
import pytest

import oracle
from paper_2410_16144_amd import synth
from test_gpu_tl2 import _quantized, codes_of_blob, dev, ops   # noqa: F401 (fixtures)

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def _differ(what, got, want):
    """'' or what differs: how many, where, by how much."""
    got, want = (np.asarray(a).astype(np.int64) for a in (got, want))
    at = np.argwhere(got != want)
    if not len(at):
        return ""
    d = (got - want)[tuple(at.T)]
    rows = np.unique(at[:, -1] if got.shape[0] == 1 else at[:, 0])
    return "%s: %d of %d differ, rows %s (blocks of 64: %s), by %s; " % (what, len(at), got.size, rows[:20].tolist(), np.unique(rows // 64)[:20].tolist(), d[:20].tolist())


@pytest.mark.parametrize("seed", range(3))
@pytest.mark.parametrize("stream", [0, 1, -1])
@pytest.mark.parametrize("N,K", [(3200, 8640), (1600, 8640), (8640, 3200), (257, 3200)])
def test_pack_and_product_each_by_itself(dev, ops, N, K, stream, seed):
    from paper_2410_16144_amd import binding
    rng = synth.rng_for(9100 + 3 * N + K + 17 * seed)
    w = synth.ternary_weights(rng, N, K, p_zero=0.4)
    bits = synth.to_bf16_bits(synth.activations(rng, 1, K, outlier_frac=0.01))
    binding.bl_set_tuning("decode_stream", stream)
    try:
        x, qa = _quantized(ops, dev, bits, K)
        pw = ops.tl2_pack(torch.from_numpy(w).to(dev), 0.02)
        _, acc = ops.tl2_gemv(pw, qa, want_acc=True)
        _, again = ops.tl2_gemv(pw, qa, want_acc=True)
        held, blob, q = (t.cpu().numpy() for t in (acc, pw.blob, qa.q))
    finally:
        binding.bl_set_tuning("decode_stream", 0)
    want_q, _, _ = oracle.quant_act(bits)
    codes, bad = oracle.tl2_encode_rows(w)
    assert bad == 0
    # the product of what the device holds, in whole numbers
    mine = (w.astype(np.int32) @ want_q[0].astype(np.int32))[None]
    said = _differ("activations", q[:, :K], want_q) + _differ("codes", codes_of_blob(blob, N, K)[:N, :(K + 2) // 3], codes) + \
        _differ("weights back", ops.tl2_unpack(pw).cpu().numpy(), w) + _differ("accumulators", held, mine) + _differ("the same launch again", again.cpu().numpy(), mine)
    assert not said, said
    assert np.array_equal(oracle.matmul_i32(want_q, w), mine)
