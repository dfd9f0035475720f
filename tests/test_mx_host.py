"""CPU checks of the 4-bit operators: sizes, refusals before anything is enqueued, and the host packer against the plain
64-bit quantiser."""
import numpy as np
import pytest

from mx_reference import E2M1, quantize, scale_at
from paper_2608_21614_b200 import inputs as gen


def test_reference_ties_and_saturation():
    x = np.zeros((1, 32))
    x[0, :10] = [4.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.9, -0.75]       # scale 1 from 7.9: ties go to even codes
    v, c, s = quantize(x)
    assert s[0, 0] == 127
    assert v[0, :10].tolist() == [4.0, 0.0, 1.0, 1.0, 2.0, 2.0, 4.0, 4.0, 6.0, -1.0]
    assert c[0, 9] == 8 | 2


def test_sizes_and_host_side_refusals():
    from paper_2608_21614_b200 import binding as B
    assert B.saem_mx_codes_bytes(3, 33) == 3 * 2 * 16 and B.saem_mx_scales_bytes(3, 33) == 512
    assert B.saem_mx_codes_bytes(0, 5) == 0 and B.saem_mx_codes_bytes(-1, 5) == 0 and B.saem_mx_codes_bytes(5, 0) == 0
    assert B.saem_mx_scales_bytes(129, 129) == 4 * 512
    assert B.saem_mx_linear_workspace_bytes(3, 33) >= 256 + 96 + 512
    cfg = B.make_config(256, 384, 8, 2, 4, ffn_path=B.SAEM_FFN_MX)
    assert B.saem_slot_bytes(cfg) == (3 * 1 * 2 + 2 * 2) * 17408                # blocks of 128 x 256: gate and up, then down
    assert B.saem_slot_bytes(B.make_config(2048, 768, 128, 8, 8, ffn_path=B.SAEM_FFN_MX)) == 3 * 2048 * 768 * 17 // 32
    assert B.saem_slot_bytes(B.make_config(256, 384, 8, 2, 4, ffn_path=6)) == 0
    P = 4096                                                                    # an address that is never read
    code = lambda f, *a: f(*a, stream=0, check=False)                          # noqa: E731
    q = lambda x, dt, r, c, st, co=P, sc=P: code(B.saem_mx_quantize, x, dt, r, c, st, co, sc)     # noqa: E731
    assert q(P, 2, 1, 32, 32) == B.SAEM_ERR_INVALID_ARG and q(None, 0, 1, 32, 32) == B.SAEM_ERR_INVALID_ARG
    assert q(P, 0, 2, 32, 31) == B.SAEM_ERR_SHAPE and q(P, 0, -1, 32, 32) == B.SAEM_ERR_SHAPE and q(P, 0, 1, 0, 32) == B.SAEM_ERR_SHAPE
    assert q(P + 1, 0, 1, 32, 32) == B.SAEM_ERR_ALIGNMENT and q(P, 0, 1, 32, 32, P + 8) == B.SAEM_ERR_ALIGNMENT
    assert q(None, 0, 0, 32, 32, None, None) == B.SAEM_OK
    d = lambda out, dt, r, c, st: code(B.saem_mx_dequantize, P, P, r, c, out, dt, st)              # noqa: E731
    assert d(P, 5, 1, 32, 32) == B.SAEM_ERR_INVALID_ARG and d(P, 1, 2, 32, 8) == B.SAEM_ERR_SHAPE
    assert d(P + 1, 1, 1, 32, 32) == B.SAEM_ERR_ALIGNMENT and d(None, 1, 0, 32, 32) == B.SAEM_OK
    m = lambda m, n, k, out=P, dt=0, st=1 << 20, w=P: code(B.saem_mx_matmul, P, P, m, w, P, n, k, out, dt, st, None)   # noqa: E731
    assert m(1, 1, 0) == m(-1, 1, 32) == m(1, 0, 32) == m((1 << 23) + 1, 1, 32) == B.SAEM_ERR_SHAPE
    assert m(2, 64, 32, st=63) == B.SAEM_ERR_SHAPE and m(1, 1, 32, dt=3) == B.SAEM_ERR_INVALID_ARG
    assert m(1, 1, 32, out=None) == B.SAEM_ERR_INVALID_ARG and m(1, 1, 32, w=P + 8) == B.SAEM_ERR_ALIGNMENT
    assert m(1, 1, 32, out=P + 2) == B.SAEM_ERR_ALIGNMENT and m(0, 1, 32, out=None) == B.SAEM_OK
    lin = lambda ws, size, dt=0: code(B.saem_mx_linear, P, dt, 4, 64, P, P, 8, 64, P, 0, 8, ws, size)   # noqa: E731
    need = B.saem_mx_linear_workspace_bytes(4, 64)
    assert lin(P, need - 1) == B.SAEM_ERR_WORKSPACE and lin(P + 16, need) == B.SAEM_ERR_ALIGNMENT
    assert lin(None, need) == B.SAEM_ERR_INVALID_ARG and lin(P, need, dt=7) == B.SAEM_ERR_INVALID_ARG
    pack = lambda c, p=P: code(B.saem_mx_pack_expert, c, P, P, P, P, P, P, p)                       # noqa: E731
    assert pack(B.make_config(256, 384, 8, 2, 4)) == B.SAEM_ERR_UNSUPPORTED
    assert pack(cfg, None) == B.SAEM_ERR_INVALID_ARG and pack(cfg, P + 8) == B.SAEM_ERR_ALIGNMENT
    assert pack(B.make_config(200, 384, 8, 2, 4, ffn_path=B.SAEM_FFN_MX)) == B.SAEM_ERR_SHAPE


def test_block_norm_refusals():
    from paper_2608_21614_b200 import binding as B
    P = 4096

    def call(x=P, y=P, gate=None, w_post=P, w_pre=P, x_out=P, n_out=P, **kw):
        c = dict(rows=2, cols=64, x_stride=64, y_stride=64, x_out_stride=64, n_stride=64, gate_stride=64, eps=1e-6)
        c.update(kw)
        return B.saem_block_norm(B.saem_norm_config(**c), x, y, gate, w_post, w_pre, x_out, n_out, stream=0, check=False)

    assert call(x_dtype=2) == call(gate_mode=4) == call(gate_mode=-1) == call(eps=-1.0) == B.SAEM_ERR_INVALID_ARG
    assert call(eps=float("nan")) == B.SAEM_ERR_INVALID_ARG
    assert call(cols=0) == call(cols=16385, x_stride=1 << 15) == call(rows=-1) == B.SAEM_ERR_SHAPE
    assert call(x_stride=63) == call(y_stride=63) == call(x_out_stride=63) == call(n_stride=0) == B.SAEM_ERR_SHAPE
    assert call(gate=P, gate_mode=B.SAEM_GATE_FULL, gate_stride=63) == B.SAEM_ERR_SHAPE
    assert call(gate=P) == call(gate_mode=B.SAEM_GATE_TOKEN) == B.SAEM_ERR_INVALID_ARG
    assert call(y=None) == call(y=None, x_out=None) == B.SAEM_ERR_INVALID_ARG                  # w_post, x_out without y
    assert call(x_out=None, n_out=None, w_pre=None) == call(n_out=None) == call(x=None) == B.SAEM_ERR_INVALID_ARG
    assert call(x=P + 2) == call(y=P + 1, y_dtype=1) == B.SAEM_ERR_ALIGNMENT
    assert call(rows=0, x=None) == B.SAEM_OK


@pytest.mark.parametrize("d,f", [(128, 128), (256, 384)])
def test_host_packer_holds_the_quantised_matrices(d, f):
    from paper_2608_21614_b200 import binding as B
    rng = np.random.default_rng(d + f)
    mats = gen.expert_weights(rng, d, f)
    mats[0][0, :32] = 0                                                         # a block of zeros
    mats[1][1, 5] = 0x7F80                                                      # an infinity: its block becomes NaN
    mats[2][3, 40] = 0x0001                                                     # a subnormal beside larger values
    cfg = B.make_config(d, f, 1, 1, 4, ffn_path=B.SAEM_FFN_MX)
    packed = np.zeros(B.saem_slot_bytes(cfg), np.uint8)
    B.saem_pack_expert_host(cfg, *mats, packed)
    blocks = packed.reshape(-1, 17408)
    chunks = lambda n: (n + 255) // 256                                          # noqa: E731
    n_gu = (f // 128) * chunks(d) * 2
    assert len(blocks) == n_gu + (d // 128) * chunks(f)
    for which, m in enumerate(mats):
        _, codes, scales = quantize(gen.bf16_bits_to_f32(m))
        K = m.shape[1]
        for row in range(m.shape[0]):
            tile, r = divmod(row, 128)
            for c in range(chunks(K)):
                b = blocks[(tile * chunks(K) + c) * 2 + which] if which < 2 else blocks[n_gu + tile * chunks(K) + c]
                want = np.zeros(256, np.int64)
                part = codes[row, c * 256:(c + 1) * 256]
                want[:len(part)] = part
                got = b[r * 128:(r + 1) * 128].reshape(8, 16)[np.arange(8) ^ (r & 7)].reshape(-1)
                assert np.array_equal(got & 15, want[0::2]) and np.array_equal(got >> 4, want[1::2]), (which, row, c)
                s = np.zeros(8, np.int64)
                s[:len(part) // 32] = scales[row, c * 8:(c + 1) * 8]
                piece = b[16384:].reshape(2, 512)[:, (r % 32) * 16 + (r // 32) * 4:][:, :4]
                assert np.array_equal(piece.reshape(-1), s), (which, row, c)


def test_scale_offsets_cover_a_piece_once():
    at = scale_at(256, 8).ravel()
    assert np.array_equal(np.sort(at), np.arange(256 * 8))
    assert len(E2M1) == 8
