"""Pins of the decode oracle: the cached-row format, its rounding, and attention over cached segments against
the oracles that already exist or closed forms."""
import numpy as np
import pytest
import torch

from oracle import decode as D


def test_row_format_round_trip_and_hand_worked_bytes():
    rng = np.random.default_rng(0)
    codes = rng.integers(-8, 8, size=512)
    byte = rng.integers(0, 255, size=32).astype(np.uint8)
    rope = rng.integers(0, 0x7F00, size=64).astype(np.uint16)
    u = D.pack_row(codes, byte, rope)
    c, b, r = D.unpack_row(u)
    assert np.array_equal(c, codes) and np.array_equal(b, byte) and np.array_equal(r, D.bf16_values(rope))
    cache = D.Cache(2)
    cache.write_row(1, 5, u)
    got = cache.rows([1], 6)[5]
    assert np.array_equal(got[:512], D.latent_values(codes[None], byte[None])[0]) and np.array_equal(got[512:], r)
    z = np.zeros(512, dtype=np.int64)
    z[0], z[1], z[2], z[33] = 7, -7, 1, -1
    u = D.pack_row(z, np.full(32, 160, np.uint8), np.zeros(64, np.uint16))
    # word 0 of unit 0: dim 0 in bits 0-3 (15), dim 1 in bits 16-19 (1), dim 2 in bits 4-7 (9), the rest 8
    assert u[0, :4].view(np.uint32)[0] == 0x8881889F
    assert u[1, :4].view(np.uint32)[0] == 0x88878888
    assert D.SCALES[160] == 1.0 and D.SCALES[0] == 2.0 ** -20 and D.SCALES[254] == 3584.0


def test_stored_values_are_bf16_numbers():
    n = np.arange(-8, 8)[:, None] * D.SCALES[None, :]
    assert np.array_equal(D.bf16_values(D.bf16_bits(n)), n)


def test_scale_and_code_rounding():
    c = np.zeros((6, 512))
    c[0, :16] = 7.0 * 1.0625                       # the scale is midway between 1 (even byte 160) and 1.125: even
    c[1, :16] = 7.0 * 1.1875                       # midway between 1.125 (161) and 1.25 (162): even is above
    c[2, 0], c[2, 1], c[2, 2] = 7.0, 2.5, 3.5      # scale 1: halves go to the even code
    c[3, 0] = 1e30                                 # beyond the largest scale: limited to 7 * 3584
    c[4, 0] = 1e-30                                # below the smallest: 0
    c[5, 0], c[5, 16] = np.inf, 1.0                # a non-finite group, its neighbour untouched
    codes, byte = D.quantise_latent(c)
    assert byte[0, 0] == 160 and byte[1, 0] == 162
    assert codes[2, :3].tolist() == [7, 2, 4]
    v = D.latent_values(codes, byte)
    assert v[3, 0] == 7 * 3584 and v[4, 0] == 0
    assert np.isnan(v[5, :16]).all() and byte[5, 0] == 255 and v[5, 16] == 7 * 0.140625 and (v[5, 17:] == 0).all()
    # every error is at most half a step, and the step is within 1/16 of max|c| / 7
    x = np.random.default_rng(1).standard_normal((200, 512))
    codes, byte = D.quantise_latent(x)
    s = np.repeat(D.SCALES[byte], 16, axis=1)
    assert (np.abs(D.latent_values(codes, byte) - x) <= 0.5 * s * (1 + 1e-12)).all()
    m = np.abs(x.reshape(200, 32, 16)).max(axis=2) / 7
    assert (np.abs(D.SCALES[byte] - m) <= m / 16 * (1 + 1e-12)).all()


def test_turn_matches_the_online_oracle():
    import oracle
    rng = np.random.default_rng(2)
    x = rng.standard_normal((5, 64))
    got = D.turn(x, np.full(5, 1234.0), 10000.0)
    back = D.turn(got, np.full(5, -1234.0), 10000.0)
    assert np.abs(back - x).max() < 1e-12
    j = 3
    a = 1234.0 * 10000.0 ** (-2 * j / 64)
    assert np.allclose(got[:, 6], x[:, 6] * np.cos(a) - x[:, 7] * np.sin(a), atol=1e-12)


def test_attention_is_dense_attention_in_one_frame():
    """Relocated segments give what one frame with keys turned to their request positions gives."""
    rng = np.random.default_rng(3)
    raw = [rng.standard_normal((n, 576)) for n in (7, 1, 20)]
    delta = [9, 0, 30]
    q = rng.standard_normal((4, 576))
    pos = np.array([49, 33, 8, -1])
    items = []
    for r, d in zip(raw, delta):
        k = r.copy()
        k[:, 512:] = D.turn(r[:, 512:], np.arange(len(r)), 10000.0)
        items.append((k, d))
    o, lse, _, _, _ = D.attention(q, pos, items, 0.07, 10000.0)
    keys = np.concatenate([np.concatenate([r[:, :512], D.turn(r[:, 512:], d + np.arange(len(r)), 10000.0)], axis=1)
                           for r, d in zip(raw, delta)])
    kp = np.concatenate([d + np.arange(len(r)) for r, d in zip(raw, delta)])
    for i in range(3):
        s = np.where(kp <= pos[i], keys @ q[i] * 0.07, -np.inf)
        w = np.exp(s - s.max())
        assert np.allclose(o[i], (w / w.sum()) @ keys[:, :512], atol=1e-12)
        assert abs(lse[i] - (s.max() + np.log(w.sum()))) < 1e-12
    assert (o[3] == 0).all() and np.isneginf(lse[3])


def test_weight_rounding():
    w = np.zeros((1, 64))
    w[0, 0], w[0, 1], w[0, 2] = 7.0, 2.5, -3.5
    assert D.quantise_weights(w, 32)[0, :3].tolist() == [7.0, 2.0, -4.0]
    assert (D.quantise_weights(np.zeros((2, 64)), 64) == 0).all()


def test_bf16_helpers_agree_with_torch():
    x = np.random.default_rng(4).standard_normal(1000) * 10.0 ** np.random.default_rng(5).integers(-8, 8, 1000)
    t = torch.from_numpy(x.astype(np.float32)).to(torch.bfloat16)
    assert np.array_equal(D.bf16_values(D.bf16_bits(x)), t.double().numpy())


def test_decode_calls_refuse_null_and_wrong_tensors_without_a_device():
    from paper_2609_07008_b200 import build
    build.build_library()
    from paper_2609_07008_b200 import binding as rk
    L = rk.lib
    assert L.rk_cache4_append(None, None, 0, None, None, 512, None, 64, None, 0, None) == 1
    assert L.rk_cache4_read(None, None, 0, None, None, 0, None, None) == 1
    assert L.rk_decode_plan(None, None, None, 0, None, None, None, None, None, 0, None) == 1
    assert L.rk_decode_plan_bytes(None, None, None) == 1
    assert L.rk_cache4_attn(None, None, None, 0, None, 0, None, None, None, None, 0, None) == 1
    assert L.rk_cache4_attn_workspace_bytes(None, None, None) == 1
    assert L.rk_quant4(None, None, None, None) == 1
    assert L.rk_matvec4(None, None, None, 0, 0, None, 0, 0, None) == 1
    i32 = torch.zeros(3, dtype=torch.int32)
    with pytest.raises(ValueError):
        rk.CacheTable(i32, torch.zeros(4, dtype=torch.int32), i32)          # host tensors
    with pytest.raises(TypeError):
        rk.CacheTable(i32.long(), i32, i32)
