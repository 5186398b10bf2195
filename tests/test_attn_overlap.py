"""Outputs that overlap an input are refused before anything is enqueued (no GPU needed)."""
import ctypes

from paper_1907_00641_amd import binding as B
from test_attn_host import BAD, FAKE, L, attn_desc  # noqa: F401


def at(p, off):
    return ctypes.c_void_p(p.value + off)


def test_attention_outputs_over_small_inputs(L):
    """lambda, lengths and mask, of which one byte is enough."""
    d = ctypes.byref(attn_desc())  # 2 sequences, 4 heads, 5 queries, 6 keys, bf16
    q, k, v, lam, ql, kl, mask, out, so, lse = FAKE[:10]
    small = {"lambda": at(lam, 7), "q_len": at(ql, 7), "k_len": at(kl, 0), "key_mask": at(mask, 11)}
    for name, p in small.items():
        assert L.pam_diff_attn_fwd(d, q, k, v, lam, ql, kl, mask, p, None, None, None, None) == BAD, name
        assert "overlaps an input" in B.last_error()
        assert L.pam_diff_attn_fwd(d, q, k, v, lam, ql, kl, mask, out, p, lse, None, None) == BAD, name
        assert "overlaps an input" in B.last_error()
        good = [q, k, v, lam, ql, kl, mask, so, lse, FAKE[10], (ctypes.c_int64 * 3)(320, 64, 16), *FAKE[11:16], None]
        for i in (11, 12, 13, 14, 15):
            args = list(good)
            args[i] = at(p, 0) if i != 15 else ctypes.c_void_p(p.value // 16 * 16)
            assert L.pam_diff_attn_bwd(d, *args) == BAD, (name, i)
            assert "overlaps an input" in B.last_error(), (name, i)


def test_rotary_outputs_over_table_and_positions(L):
    d = ctypes.byref(B.RotaryDesc(1, 1, 3, 2, 1, 8, 4, 0, 0, 9, (48, 16, 8), (24, 8, 8)))
    q, k, t, p, qo, ko = FAKE[:6]
    for bad in (at(t, 9 * 4 * 8 - 8), at(p, 8)):
        for args in ((q, k, t, p, bad, ko), (q, k, t, p, qo, bad)):
            assert L.pam_rotary(d, *args, None) == BAD
            assert "overlaps the table or pos" in B.last_error()
    f = FAKE
    for bad in (at(f[0], 24), at(f[1], 4 * 2 * 4 - 8), at(f[2], 8)):
        assert L.pam_rotary_table(f[0], f[1], f[2], 4, 4, 2, 1.0, bad, None) == BAD
        assert "overlaps an input" in B.last_error()


def test_norm_outputs_over_vectors(L):
    d = ctypes.byref(B.NormDesc(2, 0, 6, 16, 1e-6, 2, 16, 16, 0.1, 1, 1))
    x, z, wq, bq, g, sc, wp, bp, r, h, gr, gh, gx, gz, o, ws = FAKE
    for name, p in {"w_post": wq, "b_post": bq, "gate": g, "scale": sc, "w_pre": wp, "b_pre": bp}.items():
        for args in ((x, z, wq, bq, g, sc, wp, bp, at(p, 60), h), (x, z, wq, bq, g, sc, wp, bp, r, at(p, 60))):
            assert L.pam_norm_gate_fwd(d, *args, None) == BAD, name
            assert "overlaps the gate or a vector" in B.last_error(), name
    for name, p in {"w_post": wq, "b_post": bq, "gate": g, "scale": sc, "w_pre": wp}.items():
        good = [x, z, wq, bq, g, sc, wp, gr, gh] + [None] * 8 + [ws]
        for i in range(9, 18):
            args = list(good)
            args[i] = p
            assert L.pam_norm_gate_bwd(d, *args, None) == BAD, (name, i)
            assert "overlaps an input" in B.last_error(), (name, i)
