"""MI355X-native parameter-server hot path of arxiv 2406.05546 (worker CNN gradients on stale
snapshots + sync / async / stateless-buffered apply), and the dense layers and the AdamW step that larger models
trained the same way need (`dense`; `mlp` trains one with them).  The HIP library is loaded on first use of `binding` or `dense`; importing the package itself (e.g. for `synth`) does not need it."""

__all__ = ["binding", "dense", "mlp", "synth", "replay"]
